"""The 4-bit key/value cache on the GPU against tests/kv_ref.py: tables, append, read, attention, and a run of them together."""
import numpy as np
import pytest
import torch

import kv_ref as ref
import paper_2410_09687_b200 as moin
from gpu_util import kernel_launches

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def i32(a):
    return torch.as_tensor(np.ascontiguousarray(a, np.int32)).to(DEV)


# ------------------------------------------------------------------------------------------------------------- tables
def _state(rng, n_rows, max_pages, n_pages, page, fill):
    """Tables in the middle of serving: some rows hold pages, the rest of the pool is on the stack."""
    ids = list(rng.permutation(n_pages))
    table = rng.integers(-5, n_pages + 5, (n_rows, max_pages)).astype(np.int64)
    lens = np.zeros(n_rows, np.int64)
    for r in range(n_rows):
        want = int(rng.integers(0, max_pages * page + 1)) if rng.random() < fill else 0
        k = min(-(-want // page), len(ids))
        lens[r] = min(want, k * page)
        table[r, :k] = [ids.pop() for _ in range(k)]
    stack = rng.integers(0, n_pages, n_pages).astype(np.int64)
    stack[:len(ids)] = ids
    return table, stack, lens, len(ids)


def _check_update(state, want, rows, page, T, in_place):
    table, stack, lens, n_free = state
    expect = ref.update(table, stack, lens, n_free, want, rows, page, T)
    tb = moin.KvTables(i32(table), i32(stack), page, i32(lens), i32([n_free]))
    batch = moin.KvBatch(len(want), T, DEV)
    lens_out, free_out = (None, None) if in_place else (i32(lens), i32([-7]))
    for _ in range(1 if in_place else 2):     # out of place the call can be made again
        moin.kv_update(tb, i32(want), batch, rows=None if rows is None else i32(rows), lens_out=lens_out, n_free_out=free_out)
        got = {"lens": tb.lens if in_place else lens_out, "n_free": tb.n_free if in_place else free_out, "refused": batch.refused,
               "cu_q": batch.cu_q, "kv_len": batch.kv_len, "slot": batch.slot, "pos": batch.pos}
        for name, t in got.items():
            assert np.array_equal(t.cpu().numpy(), expect[name]), name
        # entries of pages that nobody holds mean nothing on the stack; held and free ones have to be right
        n, e = tb.free_pages.cpu().numpy(), expect["free_pages"]
        top = int(expect["n_free"][0])
        assert np.array_equal(n[:top], e[:top])
        assert np.array_equal(tb.block_table.cpu().numpy(), expect["block_table"])
    if not in_place:
        assert np.array_equal(tb.lens.cpu().numpy(), lens) and int(tb.n_free) == n_free


@pytest.mark.parametrize("seed", range(12))
def test_update_random(seed):
    rng = np.random.default_rng(seed)
    page = int(rng.choice([16, 32, 64, 128]))
    n_rows, max_pages = int(rng.integers(1, 90)), int(rng.integers(1, 20))
    n_pages = int(rng.integers(1, n_rows * max_pages + 2))
    state = _state(rng, n_rows, max_pages, n_pages, page, 0.7)
    R = int(rng.integers(1, n_rows + 1))
    rows = rng.permutation(n_rows)[:R]
    want = np.where(rng.random(R) < 0.25, 0, state[2][rows] + rng.integers(-3 * page, 4 * page, R))
    want = np.clip(want, 0, None)
    T = int(np.maximum(want - state[2][rows], 0).sum()) + int(rng.integers(-page, page))
    _check_update(state, want, rows, page, max(T, 0), bool(seed % 2))


def test_update_names_that_cannot_be():
    rng = np.random.default_rng(5)
    state = _state(rng, 12, 6, 60, 16, 0.8)
    rows = np.array([3, -1, 4, 12, 3, 5, 2 ** 31 - 1, 6, 7, 8])      # 3 twice, three that are not there
    want = np.array([40, 10, 6 * 16, 5, 41, -1, 1, 6 * 16 + 1, 2 ** 31 - 1, 17])
    _check_update(state, want, rows, 16, 200, False)
    state[2][4] = -3                                                    # a length that cannot be
    state[2][8] = 6 * 16 + 1
    _check_update(state, want, rows, 16, 200, True)


def test_update_pages_run_out_and_come_back_in_the_same_call():
    page, table = 16, np.zeros((5, 4), np.int64)
    table[0, :3], table[1, :2] = [4, 2, 0], [1, 3]
    state = (table, np.array([9, 9, 9, 9, 9]), np.array([45, 20, 0, 0, 0]), 0)
    # row 2 wants what row 0 gives back; row 3 wants a page more than there is, row 4 none
    _check_update(state, [0, 20, 40, 16, 0], None, page, 100, False)
    _check_update(state, [45, 33, 16, 0, 0], None, page, 100, False)
    _check_update(state, [33, 0, 0, 64, 1], None, page, 100, True)


@pytest.mark.parametrize("R,n_rows,new,page", [(1, 1, 1, 16), (1025, 1300, 1, 64), (2500, 2500, 3, 16), (60, 64, 700, 32), (3, 65536, 3000, 128)])
def test_update_sizes(R, n_rows, new, page):
    """More requests than one chunk of threads; more tokens than the first kernel places; the largest table."""
    rng = np.random.default_rng(R)
    max_pages = 4000 // page
    lens = np.zeros(n_rows, np.int64)
    rows = rng.permutation(n_rows)[:R] if R != n_rows else None
    at = np.arange(R) if rows is None else rows
    lens[at] = rng.integers(0, 300, R)
    want = np.where(rng.random(R) < 0.1, 0, lens[at] + new)
    held = -(-lens // page)
    n_pages = int(held.sum() + (-(-want // page)).sum()) - R // 3     # not enough for all
    ids = rng.permutation(n_pages)
    table = np.zeros((n_rows, max_pages), np.int64)
    o = 0
    for r in np.nonzero(held)[0]:
        table[r, :held[r]] = ids[o:o + held[r]]
        o += held[r]
    stack = np.zeros(n_pages, np.int64)
    stack[:n_pages - o] = ids[o:]
    T = int(np.maximum(want - lens[at], 0).sum()) + 5
    _check_update((table, stack, lens, n_pages - o), want, rows, page, T, False)


def test_update_without_requests_or_tokens():
    state = (np.zeros((2, 2), np.int64), np.arange(4), np.array([3, 4]), 2)
    _check_update(state, np.zeros(0, np.int64), None, 16, 5, False)
    _check_update(state, [2, 4], None, 16, 0, True)
    _check_update(state, [4, 4], None, 16, 0, True)       # no room for the token


def test_empty_tables_hand_out_pages_in_order():
    tb = moin.KvTables.empty(3, 4, 10, 32, DEV)
    b = moin.kv_update(tb, i32([33, 0, 1]), moin.KvBatch(3, 34, DEV))
    assert tb.block_table.cpu()[0, :2].tolist() == [0, 1] and int(tb.block_table[2, 0]) == 2 and int(tb.n_free) == 7
    assert b.slot.cpu().tolist() == list(range(33)) + [64] and b.cu_q.cpu().tolist() == [0, 33, 33, 34]


# ------------------------------------------------------------------------------------------------------ append and read
def _rows(rng, T, H, D):
    x = rng.standard_normal((T, H, D)) * 10.0 ** rng.integers(-3, 3, (T, H, 1)) + rng.standard_normal((T, H, 1))
    return ref.bf16(x.astype(np.float32))


def _dev(x):
    return torch.from_numpy(x).to(torch.bfloat16).to(DEV)


SLOTS = {   # distinct, as the call asks for
    "one": lambda rng, n, P: rng.integers(0, n * P, 1),
    "scattered": lambda rng, n, P: rng.permutation(n * P)[:37],
    "chunk": lambda rng, n, P: np.arange(5, min(n * P, 5 + 70)),
    "ragged": lambda rng, n, P: np.concatenate([np.arange(0, 16), [-1], np.arange(19, 31), np.arange(3 * P, 3 * P + 16), [n * P, 2 ** 31 - 1, -2 ** 31],
                                                [2 * P + 15, 2 * P + 3]]),
    "backwards": lambda rng, n, P: np.arange(40, 0, -1),
    "all": lambda rng, n, P: np.arange(n * P),
}


@pytest.mark.parametrize("slots", SLOTS)
@pytest.mark.parametrize("H,D,page", [(1, 64, 16), (4, 64, 64), (3, 128, 32), (2, 128, 128)])
def test_append_writes_the_format_and_nothing_else(slots, H, D, page):
    rng = np.random.default_rng(len(slots) + H)
    n = 4
    slot = SLOTS[slots](rng, n, page)
    T = len(slot)
    k, v = _rows(rng, T, H, D), _rows(rng, T, H, D)
    start = rng.integers(0, 256, (n, H, page // 16, D // 64, 1152)).astype(np.uint8)
    expect = start.copy()
    ref.store(expect, slot, k, 0)
    ref.store(expect, slot, v, 1)
    cache = moin.KvCache(torch.from_numpy(start.copy()).to(DEV))
    moin.kv_append(cache, i32(slot), _dev(k), _dev(v))
    assert np.array_equal(cache.pages.cpu().numpy(), expect)
    # and back: exactly the values that the codes stand for, zeros without a slot
    rk, rv = moin.kv_read(cache, i32(slot))
    for got, x in ((rk, k), (rv, v)):
        want = ref.bf16(ref.values(x.reshape(T, H, D // 64, 64)).astype(np.float32)).reshape(T, H, D)
        want[(slot < 0) | (slot >= n * page)] = 0
        assert np.array_equal(got.float().cpu().numpy(), want)


@pytest.mark.parametrize("T", [2047, 2049, 5000])
@pytest.mark.parametrize("D", [64, 128])
def test_append_many(T, D):
    """Both sizes of the window that warps look for groups in; prompts that begin inside a tile."""
    rng = np.random.default_rng(T)
    H, page, n = 2, 32, T // 32 + 300
    order, slot, left = list(rng.permutation(n)), [], T
    while left:
        m = min(left, int(rng.integers(1, 400)))
        pages = [order.pop() for _ in range(-(-(m + 40) // page)) if order]
        first = int(rng.integers(0, 40))
        run = np.concatenate([np.arange(p * page, (p + 1) * page) for p in pages])[first:first + m]
        slot.append(run)
        left -= len(run)
    slot = np.concatenate(slot)
    k, v = _rows(rng, T, H, D), _rows(rng, T, H, D)
    cache = moin.KvCache(torch.zeros(n, H, page // 16, D // 64, 1152, dtype=torch.uint8, device=DEV))
    moin.kv_append(cache, i32(slot), _dev(k), _dev(v))
    pages = cache.pages.cpu().numpy()
    for kv, x in ((0, k), (1, v)):
        c, s, z = ref.load(pages, slot, kv)
        qc, qs, qz = ref.quantise(x.reshape(T, H, D // 64, 64))
        assert np.array_equal(c, qc) and np.array_equal(s, qs) and np.array_equal(z, qz)
    rk, rv = moin.kv_read(cache, i32(slot))
    assert np.array_equal(rv.float().cpu().numpy(), ref.bf16(ref.values(v.reshape(T, H, -1, 64)).astype(np.float32)).reshape(T, H, D))
    assert np.array_equal(rk.float().cpu().numpy(), ref.bf16(ref.values(k.reshape(T, H, -1, 64)).astype(np.float32)).reshape(T, H, D))


@pytest.mark.parametrize("T,H,D,single", [(1500, 4, 64, True), (4100, 4, 64, True), (16500, 5, 64, False), (14100, 8, 128, False), (9000, 3, 128, True)])
def test_append_windows(T, H, D, single):
    """Every number of rows that a CTA looks for groups in: single tokens in pages of their own, prompts that begin inside a tile."""
    rng = np.random.default_rng(T)
    page, n = 16, (T if single else T // 16 + 200)
    if single:
        slot = rng.permutation(n) * page + rng.integers(0, page, n)
    else:
        lens = [int(x) for x in rng.integers(1, 900, 60)]
        order, slot = list(rng.permutation(n)), []
        for m in lens:
            first = int(rng.integers(0, page))
            run = np.concatenate([np.arange(p * page, (p + 1) * page) for p in [order.pop() for _ in range(-(-(m + first) // page))]])[first:first + m]
            slot.append(run)
            if sum(map(len, slot)) >= T:
                break
        slot = np.concatenate(slot)[:T]
        slot = np.concatenate([slot, np.full(T - len(slot), -1)])
    k, v = _rows(rng, T, H, D), _rows(rng, T, H, D)
    cache = moin.KvCache(torch.zeros(n, H, 1, D // 64, 1152, dtype=torch.uint8, device=DEV))
    moin.kv_append(cache, i32(slot), _dev(k), _dev(v))
    pages, at = cache.pages.cpu().numpy(), np.nonzero(slot >= 0)[0]
    for kv, x in ((0, k), (1, v)):
        c, s, z = ref.load(pages, slot[at], kv)
        qc, qs, qz = ref.quantise(x[at].reshape(len(at), H, D // 64, 64))
        assert np.array_equal(c, qc) and np.array_equal(s, qs) and np.array_equal(z, qz)
    for got, x in zip(moin.kv_read(cache, i32(slot)), (k, v)):
        want = ref.bf16(ref.values(x.reshape(T, H, D // 64, 64)).astype(np.float32)).reshape(T, H, D)
        want[slot < 0] = 0
        assert np.array_equal(got.float().cpu().numpy(), want)


@pytest.mark.parametrize("D", [64, 128])
def test_append_rotates_at_the_position(D):
    rng = np.random.default_rng(D)
    H, page, n, T = 3, 16, 12, 50
    slot = rng.permutation(n * page)[:T]
    pos = rng.integers(0, 300, T)
    pos[7], pos[20], pos[21] = -1, 300, 2 ** 31 - 1      # not in the table: skipped
    table = moin.rope_table(300, D, 10000.0, DEV)
    ang = np.arange(300)[:, None] * 10000.0 ** (-np.arange(D // 2) / (D // 2))
    assert np.abs(table.double().cpu().numpy() - np.stack([np.cos(ang), np.sin(ang)], -1)).max() <= 2.0 ** -24
    k, v = _rows(rng, T, H, D), _rows(rng, T, H, D)
    keep = (pos >= 0) & (pos < 300)
    start = rng.integers(0, 256, (n, H, 1, D // 64, 1152)).astype(np.uint8)
    expect = start.copy()
    ref.store(expect, slot[keep], ref.rotate(k[keep], pos[keep], table.cpu().numpy()), 0)
    ref.store(expect, slot[keep], v[keep], 1)
    cache = moin.KvCache(torch.from_numpy(start).to(DEV))
    moin.kv_append(cache, i32(slot), _dev(k), _dev(v), pos=i32(pos), rope=table)
    assert np.array_equal(cache.pages.cpu().numpy(), expect)


def test_append_of_rows_that_lie_apart():
    """Keys and values as parts of one fused projection's rows."""
    rng = np.random.default_rng(3)
    H, D, T, page = 4, 64, 33, 16
    both = _dev(_rows(rng, T, 3 * H, D)).reshape(T, 3 * H * D)
    k, v = both[:, H * D:2 * H * D], both[:, 2 * H * D:].view(T, H, D)
    slot = i32(np.arange(T) + 3)
    one, two = (moin.KvCache(torch.zeros(3, H, 1, 1, 1152, dtype=torch.uint8, device=DEV)) for _ in range(2))
    moin.kv_append(one, slot, k, v)
    moin.kv_append(two, slot, k.contiguous(), v.contiguous())
    assert torch.equal(one.pages, two.pages)
    out = torch.full((T, 3 * H * D), 7.0, dtype=torch.bfloat16, device=DEV)
    moin.kv_read(one, slot, out[:, :H * D], out[:, H * D:2 * H * D])
    rk, rv = moin.kv_read(one, slot)
    assert torch.equal(out[:, :H * D], rk.view(T, -1)) and torch.equal(out[:, H * D:2 * H * D], rv.view(T, -1))
    assert (out[:, 2 * H * D:] == 7).all()
    with pytest.raises(moin.MoinError):
        moin.kv_append(one, slot, both.view(T, 3 * H, D)[:, ::3][:, :H], v)     # heads that lie apart


def test_append_of_extreme_rows():
    rng = np.random.default_rng(9)
    x = _rows(rng, 12, 1, 64)
    x[0] = 0
    x[1] = 7.25
    x[2] = -3e38
    x[3, 0, 5], x[4, 0, 6], x[5, 0, 7] = np.inf, -np.inf, np.nan
    x[6, 0, :2] = [3e38, -3e38]                     # the span is not finite
    x[7] = 1e-30 * np.arange(64)
    x[8] = ref.bf16(np.float32(1e-39) * rng.standard_normal((1, 64)).astype(np.float32))     # subnormal
    x[9] = 1 + 2.0 ** -7 * (np.arange(64) % 2)      # neighbours
    x = ref.bf16(x)
    cache = moin.KvCache(torch.zeros(1, 1, 1, 1, 1152, dtype=torch.uint8, device=DEV))
    moin.kv_append(cache, i32(np.arange(12)), _dev(x), _dev(x))
    want = ref.values(x[:, :, None])[:, :, 0]
    for kv in range(2):
        c, s, z = ref.load(cache.pages.cpu().numpy(), np.arange(12), kv)
        assert np.array_equal((z[..., None] + s[..., None] * c)[:, :, 0], want, equal_nan=True)
    assert np.isnan(want[3:7]).all() and not np.isnan(want[7:]).any() and (want[:3] == x[:3]).all()


# -------------------------------------------------------------------------------------------------------------- attention
def _serve(rng, lens, H, D, page, garbage=0xFF, rows=None, n_rows=None, spread=None):
    """A cache with lens[i] tokens for request i: (cache, tables, host copies).  Page memory starts as garbage."""
    R = len(lens)
    n_rows = n_rows or R
    rows = np.arange(R) if rows is None else rows
    max_pages = max(1, -(-max(lens) // page))
    n_pages = sum(-(-n // page) for n in lens) + 2
    ids = list(rng.permutation(n_pages))
    table = np.full((n_rows, max_pages), -1, np.int64)
    slot = []
    for i, n in enumerate(lens):
        for p in range(-(-n // page)):
            table[rows[i], p] = ids.pop()
        t = np.arange(n)
        slot.append(table[rows[i], t // page] * page + t % page)
    slot = np.concatenate(slot)
    cache = moin.KvCache(torch.full((n_pages, H, page // 16, D // 64, 1152), garbage, dtype=torch.uint8, device=DEV))
    if len(slot):
        k = ref.bf16((rng.standard_normal((len(slot), H, D)) + 0.5).astype(np.float32))
        v = rng.standard_normal((len(slot), H, D))
        if spread:
            v = v * 10.0 ** rng.uniform(-spread, spread, (len(slot), H, 1))
        moin.kv_append(cache, i32(slot), _dev(k), _dev(ref.bf16(v.astype(np.float32))))
    tables = moin.KvTables(i32(table), torch.zeros(n_pages, dtype=torch.int32, device=DEV), page)
    return cache, tables, table, slot


def _check_attention(cache, tables, table, lens, q_lens, heads, rng, rope=False, rows=None, scale=None, q_scale=1.0, max_q=None, pad=3, strided=False):
    H, D, page = cache.n_kv_heads, cache.head_dim, cache.page_tokens
    cu = np.concatenate([[0], np.cumsum(q_lens)])
    T = int(cu[-1]) + pad
    q = ref.bf16((q_scale * rng.standard_normal((T, heads, D))).astype(np.float32))
    table_d, qr = None, q
    if rope:
        table_d = moin.rope_table(tables.max_pages * page, D, 10000.0, DEV)
        pos = np.concatenate([np.arange(n - m, n) for n, m in zip(lens, q_lens)] + [np.zeros(pad, np.int64)]).astype(np.int64)
        qr = ref.rotate(q, np.clip(pos, 0, None), table_d.cpu().numpy())
    want, tol = ref.attention(cache.pages.cpu().numpy(), table, rows, cu, lens, qr, D ** -0.5 if scale is None else scale, page)
    qd = _dev(q)
    out = torch.full((T, heads, D), 9.0, dtype=torch.bfloat16, device=DEV)
    if strided:
        wide = torch.full((T, heads + 2, D), 9.0, dtype=torch.bfloat16, device=DEV)
        wide[:, 1:1 + heads] = qd
        qd = wide[:, 1:1 + heads]
        out = torch.full((T, heads + 1, D), 9.0, dtype=torch.bfloat16, device=DEV)[:, 1:]
    moin.kv_attention(cache, tables, qd, i32(cu), i32(lens), max_q or max(list(q_lens) + [1]), max(list(lens) + [1]),
                      rows=None if rows is None else i32(rows), scale=scale, rope=table_d, out=out)
    got = out.float().cpu().numpy().astype(np.float64)
    assert (got[int(cu[-1]):] == 9).all(), "rows behind the last request"
    got, want, tol = got[:int(cu[-1])], want[:int(cu[-1])], tol[:int(cu[-1])]
    assert np.array_equal(np.isnan(got), np.isnan(want))
    bad = np.abs(got - want) > tol
    assert not bad.any(), (int(bad.sum()), np.argwhere(bad)[:4], np.nanmax(np.abs(got - want) / np.maximum(tol, 1e-300)))
    return got


@pytest.mark.parametrize("H,G,D,page", [(4, 8, 64, 16), (1, 1, 64, 64), (2, 7, 64, 32), (2, 4, 128, 128), (3, 2, 128, 16), (1, 16, 64, 128), (1, 33, 64, 16)])
@pytest.mark.parametrize("q_lens", ["one", "some", "chunk"])
def test_attention(H, G, D, page, q_lens):
    rng = np.random.default_rng(H * G + D)
    lens = [1, 16, 17, 300, 63, 64, 129, 500]
    q = {"one": [1] * 8, "some": [1, 2, 5, 4, 3, 0, 1, 6], "chunk": [1, 16, 9, 40, 63, 1, 0, 33]}[q_lens]
    cache, tables, table, _ = _serve(rng, lens, H, D, page)
    _check_attention(cache, tables, table, lens, q, H * G, rng, rope=True, strided=page == 32)


def test_attention_of_empty_requests_and_unseen_positions():
    """No cached tokens; more queries than cached tokens (the first see nothing); no queries; no request at all."""
    rng = np.random.default_rng(1)
    lens = [0, 5, 40, 0, 3]
    cache, tables, table, _ = _serve(rng, lens, 2, 64, 16)
    for q in ([1, 1, 1, 1, 1], [3, 9, 50, 2, 4], [0, 0, 1, 0, 0], [0, 0, 0, 0, 0]):
        got = _check_attention(cache, tables, table, lens, q, 8, rng)
        assert (got[:q[0]] == 0).all()
        _check_attention(cache, tables, table, lens, q, 8, rng, rope=True)


def test_attention_rows_out_of_range_and_impossible_lengths():
    rng = np.random.default_rng(2)
    lens = np.array([50, 20, 33, 64])
    rows = np.array([5, 2, 0, 3])
    cache, tables, table, _ = _serve(rng, lens, 2, 64, 16, rows=rows, n_rows=7)
    _check_attention(cache, tables, table, lens, [2, 1, 3, 1], 4, rng, rope=True, rows=rows)
    q = _dev(_rows(rng, 4, 4, 64))
    good = moin.kv_attention(cache, tables, q, i32([0, 1, 2, 3, 4]), i32(lens), 1, 64, rows=i32(rows))
    for r, n in (([5, -1, 0, 7], lens), (rows, np.array([50, -1, 33, 65])), (rows, np.array([50, 2 ** 31 - 1, 33, 0]))):
        out = moin.kv_attention(cache, tables, q, i32([0, 1, 2, 3, 4]), i32(n), 1, 64, rows=i32(r))
        assert torch.equal(out[[0, 2]], good[[0, 2]]) and (out[[1, 3]] == 0).all()
    # offsets that do not fit the batch are cut to it
    out = moin.kv_attention(cache, tables, q, i32([0, 1, 2, 3, 90]), i32(lens), 1, 64, rows=i32(rows))
    assert torch.equal(out[:3], good[:3])
    moin.kv_attention(cache, tables, q, i32([-5, 1, 0, 2, 3]), i32(lens), 4, 64, rows=i32(rows))
    torch.cuda.synchronize()


@pytest.mark.parametrize("impl", [1, 2])
def test_attention_bounds_that_do_not_hold(impl):
    """More queries or tokens than the call was told: zeros for the first max_q queries, nothing written behind them, others as they are."""
    rng = np.random.default_rng(33)
    lens = [100, 90, 40, 64]
    cache, tables, table, _ = _serve(rng, lens, 2, 64, 16)
    q = _dev(_rows(rng, 12, 20, 64))
    cu = i32([0, 2, 9, 10, 12])
    moin.set_option(moin.OPT_GEMM_IMPL, impl)
    try:
        good = moin.kv_attention(cache, tables, q, cu, i32(lens), 7, 100)
        for max_q, max_kv, zero in ((3, 100, [1]), (7, 70, [0, 1]), (1, 64, [0, 1, 3])):
            out = torch.full_like(q, 9.0)
            moin.kv_attention(cache, tables, q, cu, i32(lens), max_q, max_kv, out=out)
            for i, (a, b) in enumerate(((0, 2), (2, 9), (9, 10), (10, 12))):
                if i in zero:
                    assert (out[a:min(b, a + max_q)] == 0).all() and (out[a + max_q:b] == 9).all()
                else:
                    assert (out[a:b].double() - good[a:b].double()).abs().max() <= 2.0 ** -6 * good[a:b].double().abs().max()
    finally:
        moin.set_option(moin.OPT_GEMM_IMPL, 0)


def test_attention_hides_pages_that_are_not_there():
    rng = np.random.default_rng(3)
    lens = [70, 70, 40]
    cache, tables, table, _ = _serve(rng, lens, 2, 64, 16)
    table[0, 2], table[1, :], table[2, 0] = cache.n_pages, -1, 2 ** 31 - 1
    tables.block_table.copy_(i32(table))
    got = _check_attention(cache, tables, table, lens, [1, 1, 1], 4, rng)
    assert (got[1] == 0).all()


@pytest.mark.parametrize("D", [64, 128])
def test_attention_nan_stays_where_it_is_seen(D):
    """A stored NaN (key or value) reaches the queries that see it and no other: earlier positions, other heads, other requests."""
    rng = np.random.default_rng(4)
    lens, H = [60, 40], 2
    cache, tables, table, slot = _serve(rng, lens, H, D, 16)
    k, v = _rows(rng, 2, H, D), _rows(rng, 2, H, D)
    k[0, 1, 3], v[1, 0, D - 1] = np.inf, np.nan
    at = [slot[57], slot[55]]                            # request 0, positions 57 (key, head 1) and 55 (value, head 0, last plane)
    moin.kv_append(cache, i32(at), _dev(k), _dev(v))
    got = _check_attention(cache, tables, table, lens, [8, 3], H * 2, rng)
    nan = np.isnan(got)
    assert nan[5:8, 2:].all() and not nan[:5, 2:].any()          # positions 57 .. 59 of head group 1
    assert nan[3:8, :2, -64:].all() and not nan[:3].any() and not nan[8:].any()
    if D == 128:
        assert not nan[:, :2, :64].any()


def test_attention_of_unbalanced_scales():
    """Value scales over twelve orders of magnitude, constant values, zeros, sharp and flat softmaxes."""
    rng = np.random.default_rng(6)
    lens = [500, 200, 77]
    cache, tables, table, slot = _serve(rng, lens, 2, 64, 32, spread=6)
    for q_scale in (0.01, 1.0, 30.0):
        _check_attention(cache, tables, table, lens, [1, 1, 1], 16, rng, q_scale=q_scale)
        _check_attention(cache, tables, table, lens, [9, 2, 30], 4, rng, q_scale=q_scale)
    v = np.zeros((77, 2, 64), np.float32)
    v[::3], v[1::3] = 5.0, -1e30
    moin.kv_append(cache, i32(slot[700:]), _dev(_rows(rng, 77, 2, 64)), _dev(ref.bf16(v)))
    _check_attention(cache, tables, table, lens, [1, 1, 1], 16, rng)
    for scale in (0.0, -0.3, 2.0):
        _check_attention(cache, tables, table, lens, [1, 3, 2], 2, rng, scale=scale)


# Long chunks have a kernel of their own where heads are 64 wide; here every call is made with either.
CHUNK = [40, 3, 90, 17, 65]


@pytest.fixture(params=["rows", "tcgen05"])
def kernel(request):
    moin.set_option(moin.OPT_GEMM_IMPL, 1 + (request.param == "tcgen05"))
    yield request.param
    moin.set_option(moin.OPT_GEMM_IMPL, 0)


@pytest.mark.parametrize("heads,H", [(16, 2), (14, 2), (4, 4), (150, 1)])
def test_chunks_behind_pasts(heads, H, kernel):
    rng = np.random.default_rng(heads)
    lens = [40, 300, 513, 64, 700]
    cache, tables, table, _ = _serve(rng, lens, H, 64, 32)
    q = CHUNK if heads < 100 else [2, 1, 3, 0, 2]
    _check_attention(cache, tables, table, lens, q if heads // H > 1 else [40, 190, 200, 64, 129], heads, rng, rope=True, strided=heads == 14)


def test_chunks_of_empty_requests_hidden_pages_and_unseen_positions(kernel):
    rng = np.random.default_rng(21)
    lens = [0, 20, 513, 64, 130, 0]
    cache, tables, table, _ = _serve(rng, lens, 2, 64, 16)
    table[2, 3], table[2, 4], table[2, 20], table[4, 8], table[3, :] = -1, cache.n_pages, 2 ** 31 - 1, -7, -1
    tables.block_table.copy_(i32(table))
    for q in ([5, 100, 70, 9, 64, 0], [0, 0, 128, 64, 1, 3], [0, 0, 0, 0, 129, 1], [70, 70, 70, 70, 70, 70]):
        got = _check_attention(cache, tables, table, lens, q, 16, rng, rope=True)
        assert (got[:q[0]] == 0).all()


def test_chunks_nan_stays_where_it_is_seen(kernel):
    rng = np.random.default_rng(22)
    lens, H = [200, 90], 2
    cache, tables, table, slot = _serve(rng, lens, H, 64, 16)
    k, v = _rows(rng, 3, H, 64), _rows(rng, 3, H, 64)
    k[0, 1, 3], v[1, 0, 63], v[2, 1, 0] = np.inf, np.nan, -np.inf
    at = [slot[127], slot[130], slot[200]]       # request 0: a key of head 1 at 127, a value of head 0 at 130; request 1: a value of head 1 at 0
    moin.kv_append(cache, i32(at), _dev(k), _dev(v))
    got = _check_attention(cache, tables, table, lens, [120, 90], H * 4, rng)
    nan = np.isnan(got).all(-1)
    pos = np.concatenate([np.arange(80, 200), np.arange(90)])
    first = np.arange(210) < 120
    assert np.array_equal(np.isnan(got).any(-1), nan)
    assert np.array_equal(nan[:, :4], np.repeat((first & (pos >= 130))[:, None], 4, 1))
    assert np.array_equal(nan[:, 4:], np.repeat((~first | (pos >= 127))[:, None], 4, 1))


def test_chunks_of_unbalanced_scales(kernel):
    rng = np.random.default_rng(23)
    lens = [500, 200, 77]
    cache, tables, table, slot = _serve(rng, lens, 2, 64, 32, spread=6)
    for q_scale in (0.01, 1.0, 30.0):
        _check_attention(cache, tables, table, lens, [150, 64, 77], 8, rng, q_scale=q_scale)
    v = np.zeros((77, 2, 64), np.float32)
    v[::3], v[1::3] = 5.0, -1e30
    moin.kv_append(cache, i32(slot[700:]), _dev(_rows(rng, 77, 2, 64)), _dev(ref.bf16(v)))
    _check_attention(cache, tables, table, lens, [1, 1, 77], 16, rng)
    for scale in (0.0, -0.3, 2.0):
        _check_attention(cache, tables, table, lens, [1, 30, 70], 8, rng, scale=scale)


def test_chunk_rows_do_not_reach_one_another(kernel):
    rng = np.random.default_rng(24)
    lens, G = [300], 4
    cache, tables, _, _ = _serve(rng, lens, 1, 64, 16)
    q = ref.bf16(rng.standard_normal((100, G, 64)).astype(np.float32))
    plain = moin.kv_attention(cache, tables, _dev(q), i32([0, 100]), i32(lens), 100, 300)
    changed = torch.zeros(100, G, dtype=torch.bool, device=DEV)
    for (i, h), x in {(0, 1): 1e30, (31, 2): np.nan, (32, 0): np.inf, (50, 3): 1e-30, (99, 3): -np.inf}.items():
        q[i, h, 3:] = x
        changed[i, h] = True
    out = moin.kv_attention(cache, tables, _dev(q), i32([0, 100]), i32(lens), 100, 300)
    assert torch.equal(out[~changed], plain[~changed])
    assert out[31, 2].isnan().all() and out[32, 0].isnan().all() and out[99, 3].isnan().all() and out[50, 3].isfinite().all()


def test_chunks_the_same_bits_and_beside_one_another(kernel):
    """Asked again, and with a second call on another stream at the same time; and the kernel is the one meant."""
    rng = np.random.default_rng(25)
    lens = [900, 513]
    cache, tables, table, _ = _serve(rng, lens, 2, 64, 64)
    q = _dev(ref.bf16(rng.standard_normal((104, 8, 64)).astype(np.float32)))
    args = (cache, tables, q, i32([0, 64, 104]), i32(lens), 64, 900)
    first = moin.kv_attention(*args)
    assert list(kernel_launches(lambda: moin.kv_attention(*args))) == ["kv_chunk" if kernel == "tcgen05" else "kv_attention"]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for _ in range(5):
        with torch.cuda.stream(side):
            other = moin.kv_attention(*args)
        again = moin.kv_attention(*args)
        torch.cuda.synchronize()
        assert torch.equal(again, first) and torch.equal(other, first)


@pytest.mark.parametrize("lens,q", [([3000, 2990, 17], [300, 1, 17]), ([64] * 70, [64] * 70), ([700] * 5, [129, 128, 127, 1, 64]), ([1500], [150])])
def test_chunks_of_many_items(lens, q, kernel):
    """More items than CTAs, rows of items that end in a request's last tile, the longest request first and last."""
    rng = np.random.default_rng(len(lens))
    cache, tables, table, _ = _serve(rng, lens, 1, 64, 16)
    _check_attention(cache, tables, table, lens, q, 2 if len(lens) > 9 else 3, rng, rope=True)


@pytest.mark.parametrize("kind", ["two items", "runs of requests", "one head each", "short behind long"])
def test_chunk_shares(kind, kernel):
    """Items that many CTAs share, shares that hold many items, requests without tokens, keys or queries between them."""
    rng = np.random.default_rng(27)
    if kind == "two items":
        lens, q, H, G = [9000], [200], 1, 1
    elif kind == "runs of requests":
        lens = [int(x) for x in rng.integers(0, 300, 150)]
        q, H, G = [int(rng.integers(0, min(n, 70) + 1)) for n in lens], 1, 3
    elif kind == "one head each":
        lens, q, H, G = [1, 700, 64, 2000, 65, 0, 1300], [1, 130, 64, 1, 65, 0, 128], 3, 1
    else:
        lens, q, H, G = [4000] + [20] * 30 + [2500], [3] + [20] * 30 + [129], 1, 2
    cache, tables, table, _ = _serve(rng, lens, H, 64, 64)
    _check_attention(cache, tables, table, lens, q, H * G, rng, rope=True)


def test_chunk_maxima_that_move(kernel):
    """Scores that rise by 20 powers of two from tile to tile, fall as fast, jump once, and stay: weights are taken against the largest so far."""
    rng = np.random.default_rng(28)
    lens, q_lens, heads = [1000, 500], [70, 33], 4
    cache, tables, table, slot = _serve(rng, lens, 1, 64, 64)
    u = rng.choice([-1.0, 1.0], (4, 64))
    t = np.concatenate([np.arange(n) for n in lens])
    k = 1.75 * t[:, None] / 64 * u[0] + np.where(t[:, None] >= 333, 9.0, 0.0) * u[1] + 0.1 * rng.standard_normal((len(t), 64))
    v = rng.standard_normal((len(t), 64)) + 1.0
    moin.kv_append(cache, i32(slot), _dev(ref.bf16(k[:, None].astype(np.float32))), _dev(ref.bf16(v[:, None].astype(np.float32))))
    q = ref.bf16(np.broadcast_to(np.stack([u[0], -u[0], u[1], 0.01 * u[2]]), (103, heads, 64)).astype(np.float32))
    cu = [0, 70, 103]
    want, tol = ref.attention(cache.pages.cpu().numpy(), table, None, cu, lens, q, 0.125, 64)
    got = moin.kv_attention(cache, tables, _dev(q), i32(cu), i32(lens), 70, 1000, scale=0.125).float().cpu().numpy().astype(np.float64)
    bad = np.abs(got - want) > tol
    assert not bad.any(), (int(bad.sum()), np.argwhere(bad)[:4], (np.abs(got - want) / tol).max())


def test_chunks_of_a_scale_that_vanishes(kernel):
    """Scores of 1e-40, whose factors underflow: the means of the values seen."""
    rng = np.random.default_rng(29)
    lens = [200, 90]
    cache, tables, table, _ = _serve(rng, lens, 2, 64, 16)
    _check_attention(cache, tables, table, lens, [80, 90], 8, rng, scale=1e-40)


def test_the_rule_sends_long_chunks_to_the_tensor_cores():
    rng = np.random.default_rng(26)
    cache, tables, _, _ = _serve(rng, [600, 600], 4, 64, 64)
    for n, name in ((1, "kv_attention"), (256, "kv_chunk")):
        q = _dev(ref.bf16(rng.standard_normal((2 * n, 32, 64)).astype(np.float32)))
        assert list(kernel_launches(lambda: moin.kv_attention(cache, tables, q, i32([0, n, 2 * n]), i32([600, 600]), n, 600))) == [name]


def test_attention_query_rows_do_not_reach_one_another():
    """Queries of 1e30, of 1e-30, infinite ones and NaN beside ordinary ones, in the same head group and chunk."""
    rng = np.random.default_rng(7)
    lens, H, G = [100], 1, 8
    cache, tables, _, _ = _serve(rng, lens, H, 64, 16)
    q = _rows(rng, 4, G, 64)
    q[:] = ref.bf16(rng.standard_normal(q.shape).astype(np.float32))
    plain = moin.kv_attention(cache, tables, _dev(q), i32([0, 4]), i32(lens), 4, 100)
    q[0, 1], q[1, 2, 3], q[2, 3, 4], q[3, 0] = 1e30, np.nan, np.inf, 1e-30
    out = moin.kv_attention(cache, tables, _dev(q), i32([0, 4]), i32(lens), 4, 100)
    changed = torch.zeros(4, G, dtype=torch.bool, device=DEV)
    for i, h in ((0, 1), (1, 2), (2, 3), (3, 0)):
        changed[i, h] = True
    assert torch.equal(out[~changed], plain[~changed])
    assert out[1, 2].isnan().all() and out[2, 3].isnan().all() and out[0, 1].isfinite().all()
    # 1e-30: all scores alike, the mean of the values
    k, v = moin.kv_read(cache, tables.block_table[0].repeat_interleave(16)[:100] * 16 + torch.arange(100, dtype=torch.int32, device=DEV) % 16)
    mean = v.double().mean(0)[0]
    assert ((out[3, 0].double() - mean).abs() <= 2.0 ** -8 * mean.abs() + 2.0 ** -8 * v.double().abs().max()).all()


@pytest.mark.parametrize("lens,H,G,D", [([4096, 1, 700], 4, 8, 64), ([2500], 1, 1, 64), ([3333], 8, 4, 128), ([9, 4000, 30, 17, 2222, 1100], 2, 8, 64)])
def test_attention_long(lens, H, G, D):
    rng = np.random.default_rng(sum(lens))
    cache, tables, table, _ = _serve(rng, lens, H, D, 64)
    _check_attention(cache, tables, table, lens, [1] * len(lens), H * G, rng, rope=True)
    if G <= 4:
        _check_attention(cache, tables, table, lens, [3] * len(lens), H * G, rng)


@pytest.mark.parametrize("D,G,q", [(64, 8, 1), (64, 4, 3), (64, 4, 30), (128, 4, 1), (128, 4, 3), (128, 2, 20)])
@pytest.mark.parametrize("kind", ["one", "few long", "many short", "more than there are CTAs"])
def test_attention_splits(kind, D, G, q):
    """Whole items, equal shares and cuts of one request's items: every row block size and head width, pieces that begin and end anywhere."""
    rng = np.random.default_rng(D + G + q)
    lens = {"one": [1900], "few long": [1700, 3, 2100, 800, 16, 1601], "many short": [int(x) for x in rng.integers(1, 60, 40)],
            "more than there are CTAs": [int(x) for x in rng.integers(1, 40, 400)]}[kind]
    H = 4 if kind == "more than there are CTAs" else 2
    if kind == "more than there are CTAs" and q > 1:
        lens = lens[:130]
    cache, tables, table, _ = _serve(rng, lens, H, D, 32)
    moin.set_option(moin.OPT_GEMM_IMPL, 1)
    try:
        _check_attention(cache, tables, table, lens, [min(q, n) for n in lens], H * G, rng, rope=True)
        # told that requests may be long, the call cannot take whole items
        few = lens[:5]
        out = moin.kv_attention(cache, tables, _dev(ref.bf16(rng.standard_normal((5, H * G, D)).astype(np.float32))), i32(np.arange(len(few) + 1)), i32(few))
        assert out[:len(few)].isfinite().all()
    finally:
        moin.set_option(moin.OPT_GEMM_IMPL, 0)


def test_attention_sums_over_a_long_request_hold_their_precision():
    """131 072 tokens, a flat softmax: the result is the mean of many values and a few thousandths of them.  Error allowed: 2^-8
    of the result's size (its rounding to bf16, in norm 2^-9), and 2^-11 (rounded weights) times the largest sv c = 15 sv over the
    square root of the number of tokens (the roundings are independent)."""
    n, H, D, page = 131072, 1, 64, 128
    gen = torch.Generator(device=DEV).manual_seed(1)
    cache = moin.KvCache.empty(n // page, page, H, D, DEV)
    k = torch.randn(n, H, D, generator=gen, device=DEV).to(torch.bfloat16)
    v = torch.randn(n, H, D, generator=gen, device=DEV).to(torch.bfloat16)
    slot = torch.arange(n, dtype=torch.int32, device=DEV)
    moin.kv_append(cache, slot, k, v)
    tables = moin.KvTables(slot[:n // page].view(1, -1).contiguous(), torch.zeros(n // page, dtype=torch.int32, device=DEV), page)
    q = (0.2 * torch.randn(1, 8, D, generator=gen, device=DEV)).to(torch.bfloat16)
    out = moin.kv_attention(cache, tables, q, i32([0, 1]), i32([n]), 1, n)
    code = {kv: [torch.from_numpy(x).to(DEV) for x in ref.load(cache.pages.cpu().numpy(), np.arange(n), kv)] for kv in range(2)}
    K, V = ((z[..., None] + s[..., None] * c).reshape(n, D) for c, s, z in (code[0], code[1]))
    want = torch.softmax(q[0].double() @ K.T / 8, -1) @ V
    off, size = (out[0].double() - want).norm(), want.norm()
    assert off <= 2.0 ** -8 * size + 2.0 ** -11 * 15 * code[1][1].max() * (8 * D / n) ** 0.5, (off / size)
    assert size < 0.02 * V.norm() / n ** 0.5 * (8 * 64) ** 0.5


def test_offsets_beyond_32_bits():
    """A pool of 5.9 GB whose last pages hold the request."""
    H, D, page = 8, 128, 128
    n_pages = 40000
    cache = moin.KvCache.empty(n_pages, page, H, D, DEV)
    assert cache.pages.numel() > 2 ** 32
    rng = np.random.default_rng(8)
    n = 300
    pages = np.array([n_pages - 1, n_pages - 7, n_pages // 2 + 9000])
    t = np.arange(n)
    slot = pages[t // page] * page + t % page
    k, v = _rows(rng, n, H, D), _rows(rng, n, H, D)
    moin.kv_append(cache, i32(slot), _dev(k), _dev(v))
    rk, rv = moin.kv_read(cache, i32(slot))
    assert np.array_equal(rv.float().cpu().numpy(), ref.bf16(ref.values(v.reshape(n, H, 2, 64)).astype(np.float32)).reshape(n, H, D))
    small = moin.KvCache(cache.pages[torch.from_numpy(pages).to(DEV)].clone())
    q = _dev(_rows(rng, 1, H, D))
    big = moin.kv_attention(cache, moin.KvTables(i32(pages[None]), torch.zeros(n_pages, dtype=torch.int32, device=DEV), page), q, i32([0, 1]), i32([n]), 1, n)
    one = moin.kv_attention(small, moin.KvTables(i32([[0, 1, 2]]), torch.zeros(3, dtype=torch.int32, device=DEV), page), q, i32([0, 1]), i32([n]), 1, n)
    assert torch.equal(big, one)


def test_calls_with_other_tensors_are_refused():
    """Types, shapes, places and orders that the calls do not take: an error before anything is launched."""
    T, H, D = 5, 2, 64
    cache, tables = moin.KvCache.empty(3, 16, H, D, DEV), moin.KvTables.empty(2, 2, 3, 16, DEV)
    batch, rope = moin.KvBatch(2, T, DEV), moin.rope_table(32, D, 1e4, DEV)
    want = i32([3, 2])
    k = torch.zeros(T, H, D, dtype=torch.bfloat16, device=DEV)
    q, cu = torch.zeros(T, 4, D, dtype=torch.bfloat16, device=DEV), i32([0, 3, 5])
    moin.kv_update(tables, want, batch)
    slot, pos = batch.slot.clone(), batch.pos.clone()
    moin.kv_append(cache, slot, k, k, pos=pos, rope=rope)
    good = moin.kv_attention(cache, tables, q, cu, want, rope=rope)
    assert good.shape == q.shape
    bad = [lambda: moin.kv_update(tables, want.long(), batch), lambda: moin.kv_update(tables, want[:1], batch), lambda: moin.kv_update(tables, want.cpu(), batch),
           lambda: moin.kv_update(tables, want, batch, rows=i32([0])), lambda: moin.kv_update(tables, want, batch, lens_out=i32([0])),
           lambda: moin.kv_update(tables, want, batch, n_free_out=i32([0, 0])), lambda: moin.kv_update(tables, torch.stack([want, want], 1)[:, 0], batch),
           lambda: moin.kv_update(tables, [3, 2], batch),
           lambda: moin.kv_append(cache, slot, k.float(), k), lambda: moin.kv_append(cache, slot, k, k[:4]), lambda: moin.kv_append(cache, slot, k, k.cpu()),
           lambda: moin.kv_append(cache, slot, k.transpose(0, 1).contiguous().transpose(0, 1), k), lambda: moin.kv_append(cache, slot, k, k.view(T, D, H)),
           lambda: moin.kv_append(cache, slot.short(), k, k), lambda: moin.kv_append(cache, slot, k, k, pos=pos[:4], rope=rope),
           lambda: moin.kv_append(cache, slot, k, k, rope=rope), lambda: moin.kv_append(cache, slot, k, k, pos=pos, rope=rope.bfloat16()),
           lambda: moin.kv_append(cache, slot, k, k, pos=pos, rope=rope[:, :16]), lambda: moin.kv_append(cache, slot, torch.zeros(T, H + 1, D + 4, dtype=torch.bfloat16, device=DEV)[:, :H, :D], k),
           lambda: moin.kv_read(cache, slot.cpu()), lambda: moin.kv_read(cache, slot, k=k.half()), lambda: moin.kv_read(cache, slot, v=k[:2]),
           lambda: moin.kv_attention(cache, tables, q.float(), cu, want), lambda: moin.kv_attention(cache, tables, q.view(T, -1), cu, want),
           lambda: moin.kv_attention(cache, tables, q[:, :3].contiguous(), cu, want), lambda: moin.kv_attention(cache, tables, q, cu[:2], want),
           lambda: moin.kv_attention(cache, tables, q, cu, want.long()), lambda: moin.kv_attention(cache, tables, q, cu, want, rows=i32([0, 1, 0])),
           lambda: moin.kv_attention(cache, tables, q, cu, want, out=q[:3]), lambda: moin.kv_attention(cache, tables, q, cu, want, out=q.float()),
           lambda: moin.kv_attention(cache, tables, q, cu, want, rope=rope[:31].contiguous()),
           lambda: moin.kv_attention(cache, moin.KvTables.empty(2, 2, 3, 32, DEV), q, cu, want)]
    bad += [lambda: moin.KvCache.empty(2, 48, 1, 64, DEV), lambda: moin.KvCache.empty(2, 16, 1, 96, DEV)]
    for i, call in enumerate(bad):
        with pytest.raises(moin.MoinError):
            call()
            pytest.fail(f"call {i} went through")
    assert torch.equal(moin.kv_attention(cache, tables, q, cu, want, rope=rope), good)
    # nothing to do: no tokens, no requests
    moin.kv_append(cache, slot[:0], k[:0], k[:0])
    assert moin.kv_read(cache, slot[:0])[0].shape == (0, H, D) and moin.kv_attention(cache, tables, q[:0], i32([0]), want[:0]).shape == (0, 4, D)


# ------------------------------------------------------------------------------------------------------------ together
def _steps(rng, R, page):
    """Wanted lengths of a few steps: prompts of which one comes late, tokens one by one, a request that ends, its row reused."""
    prompt = rng.integers(1, 60, R)
    yield np.where(np.arange(R) == 2, 0, prompt)
    n = np.where(np.arange(R) == 2, 0, prompt)
    for step in range(6):
        n = n + (n > 0)
        if step == 1:
            n[2] = 37
        if step == 3:
            n[1] = 0
        if step == 4:
            n[1] = 20
        yield n.copy()


@pytest.mark.parametrize("H,G,D,page", [(2, 4, 64, 16), (1, 8, 128, 32)])
def test_generation_loop(H, G, D, page):
    """update -> append -> attention, step after step, against the tokens kept by the test."""
    rng = np.random.default_rng(H)
    R = 4
    tables = moin.KvTables.empty(R, 8, 20, page, DEV)
    cache = moin.KvCache(torch.full((20, H, page // 16, D // 64, 1152), 0xFF, dtype=torch.uint8, device=DEV))
    rope = moin.rope_table(8 * page, D, 10000.0, DEV)
    lens = np.zeros(R, np.int64)
    kept = [np.zeros((0, H, D), np.float32)] * R, [np.zeros((0, H, D), np.float32)] * R
    for want in _steps(rng, R, page):
        new = np.maximum(want - lens, 0)
        T = int(new.sum()) + 2
        q, k, v = (_rows(rng, T, h, D) for h in (H * G, H, H))
        q = ref.bf16(rng.standard_normal(q.shape).astype(np.float32))
        batch = moin.kv_update(tables, i32(want), moin.KvBatch(R, T, DEV))
        moin.kv_append(cache, batch.slot, _dev(k), _dev(v), pos=batch.pos, rope=rope)
        out = moin.kv_attention(cache, tables, _dev(q), batch.cu_q, batch.kv_len, rope=rope)
        assert int(batch.refused) == 0
        o = 0
        pages, table = cache.pages.cpu().numpy(), tables.block_table.cpu().numpy()
        pos = np.concatenate([np.arange(w - m, w) for w, m in zip(want, new)] + [[0, 0]]).astype(np.int64)
        kr, qr = ref.rotate(k, pos, rope.cpu().numpy()), ref.rotate(q, pos, rope.cpu().numpy())
        for i in range(R):
            for x, rows in zip(kept, (kr, v)):
                x[i] = np.concatenate([x[i][:want[i]], rows[o:o + new[i]]])
            if want[i]:
                t = np.arange(want[i])
                slot = table[i, t // page] * page + t % page
                for kv in range(2):
                    c, s, z = ref.load(pages, slot, kv)
                    assert np.array_equal((z[..., None] + s[..., None] * c), ref.values(kept[kv][i].reshape(-1, H, D // 64, 64)))
            o += new[i]
        expect, tol = ref.attention(pages, table, None, batch.cu_q.cpu().numpy(), want, qr, D ** -0.5, page)
        got = out.double().cpu().numpy()
        assert (np.abs(got[:o] - expect[:o]) <= tol[:o]).all()
        lens = want


def test_captured_generation():
    """A step captured once and replayed, lengths advancing on the GPU, gives what single calls give; a second graph with its own
    tables runs on another stream at the same time."""
    H, G, D, page, R = 2, 8, 64, 16, 3
    rng = np.random.default_rng(11)

    def server():
        tables = moin.KvTables.empty(R, 40, 140, page, DEV)
        cache = moin.KvCache(torch.zeros(140, H, 1, 1, 1152, dtype=torch.uint8, device=DEV))
        want = i32([500, 30, 77])
        batch = moin.KvBatch(R, 607, DEV)
        moin.kv_update(tables, want, batch)
        k = _dev(ref.bf16(np.random.default_rng(1).standard_normal((607, H, D)).astype(np.float32)))
        moin.kv_append(cache, batch.slot, k, k)
        return tables, cache, want, moin.KvBatch(R, R, DEV)

    xs = [[_dev(ref.bf16(rng.standard_normal((R, h, D)).astype(np.float32))) for h in (H * G, H, H)] for _ in range(5)]

    def step(sv, q, k, v, out):
        tables, cache, want, batch = sv
        want += 1
        moin.kv_update(tables, want, batch)
        moin.kv_append(cache, batch.slot, k, v)
        moin.kv_attention(cache, tables, q, batch.cu_q, batch.kv_len, 1, 640, out=out)

    plain, sv = [], server()
    for x in xs:
        out = torch.empty_like(x[0])
        step(sv, *x, out)
        plain.append(out)
    runs = []
    for _ in range(2):
        sv, buf, out = server(), [t.clone() for t in xs[0]], torch.empty_like(xs[0][0])
        stream = torch.cuda.Stream()
        g = torch.cuda.CUDAGraph()
        want0 = sv[2].clone()
        torch.cuda.synchronize()
        with torch.cuda.graph(g, stream=stream):
            step(sv, *buf, out)
        sv[2].copy_(want0)
        runs.append((sv, buf, out, stream, g))
    torch.cuda.synchronize()
    for i, x in enumerate(xs):
        for sv, buf, out, stream, g in runs:
            with torch.cuda.stream(stream):
                for b, t in zip(buf, x):
                    b.copy_(t)
                g.replay()
        torch.cuda.synchronize()
        for _, _, out, _, _ in runs:
            assert torch.equal(out, plain[i])


def test_same_call_same_bits():
    rng = np.random.default_rng(12)
    lens = [2000, 900, 40, 3]
    cache, tables, _, _ = _serve(rng, lens, 4, 64, 16)
    q = _dev(_rows(rng, 4, 32, 64))
    args = (cache, tables, q, i32([0, 1, 2, 3, 4]), i32(lens), 1, 2000)
    first = moin.kv_attention(*args)
    for _ in range(5):
        assert torch.equal(moin.kv_attention(*args), first)
    # alone and among others a request may be split differently: a step of the result's rounding at most
    alone = moin.kv_attention(cache, tables, q[:1], i32([0, 1]), i32(lens[:1]), 1, 2000)
    assert (alone[0].double() - first[0].double()).abs().max() <= 2.0 ** -7 * first[0].double().abs().max()
