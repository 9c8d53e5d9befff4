"""Cached attention where its numbers are large, small or many.  Reference and bounds: tests/kv_exact.py, tests/kv_ref.py."""
import numpy as np
import pytest
import torch

import kv_exact as exact
import kv_ref as ref
import paper_2410_09687_b200 as moin
from test_gpu_kv import DEV, _dev, _serve, i32

pytestmark = pytest.mark.gpu


@pytest.fixture(params=["rows", "tcgen05"])
def kernel(request):
    moin.set_option(moin.OPT_GEMM_IMPL, 1 + (request.param == "tcgen05"))
    yield request.param
    moin.set_option(moin.OPT_GEMM_IMPL, 0)


@pytest.mark.parametrize("unlike", [0, -30, 20, 60])
@pytest.mark.parametrize("D,new,beside", [(64, 1, False), (64, 5, False), (64, 70, True), (128, 1, False), (128, 9, True)])
@pytest.mark.parametrize("power", [20, 24, 27, 30, 60, 100, 116, 120])
def test_queries_near_the_largest_number(D, new, beside, power, unlike, kernel):
    """Queries of 2^20 to 2^120 against keys a_t u: the token with the largest a_t takes all weight, so the result is its value (half a
    bf16 step, and half an fp16 step of what its weight multiplies, or of weight and value where both are in fp16).  Ordinary
    queries beside them give the same bits as alone, but where tokens of unlike sizes (every seventh value 2^unlike times the others) are taken one by one."""
    rng = np.random.default_rng(power + D)
    n, H, G, page = 200, 2, 4, 16
    cache, tables, table, slot = _serve(rng, [n], H, D, page)
    u = rng.choice([-1.0, 1.0], D)
    a = rng.uniform(-3, 3, n)
    a[0], a[1] = 4, -4
    k = ref.bf16((a[:, None, None] * u).astype(np.float32)) * np.ones((1, H, 1), np.float32)
    v = ref.bf16(rng.standard_normal((n, H, D)).astype(np.float32))
    if unlike:
        v[::7] *= np.float32(2.0 ** unlike)
    moin.kv_append(cache, i32(slot), _dev(k), _dev(v))
    sign = np.where(np.arange(new * H * G).reshape(new, H * G) % 3 == 0, -1.0, 1.0)
    q = ref.bf16((2.0 ** power * sign[..., None] * u).astype(np.float32))
    big = np.ones((new, H * G), bool)
    if beside:
        big[:, ::2] = False
        q[~big] = ref.bf16(rng.standard_normal((int((~big).sum()), D)).astype(np.float32))
    args = (i32([0, new]), i32([n]), new, n)
    got = moin.kv_attention(cache, tables, _dev(q), *args)
    c, s, z = ref.load(cache.pages.cpu().numpy(), slot[:2], 1)
    val, step = ((z[..., None] + s[..., None] * c).reshape(2, H, D), (s[..., None] * c).reshape(2, H, D))
    head, at = np.arange(H * G) // G, (sign < 0).astype(int)
    want, part = val[at, head[None]], step[at, head[None]]
    tol = 2.0 ** -8 * np.abs(want) + (2.0 ** -11 * part if kernel == "rows" or D == 128 else 2.0 ** -10 * np.abs(want) + 2.0 ** -30 * np.abs(val).max((1, 2))[at][..., None])
    err = np.abs(got.double().cpu().numpy() - want)
    assert (err <= tol)[big].all(), np.nanmax(err[big])
    if beside and not unlike:
        small = q.copy()
        small[big] = 0
        alone = moin.kv_attention(cache, tables, _dev(small), *args)
        assert torch.equal(got[torch.from_numpy(~big).to(DEV)], alone[torch.from_numpy(~big).to(DEV)])


def _wide(rng, n, H, powers, page=32):
    """A request of n tokens whose value planes are multiplied with 2^powers[t][plane]."""
    cache, tables, table, slot = _serve(rng, [n], H, 128, page)
    k = ref.bf16(rng.standard_normal((n, H, 128)).astype(np.float32))
    v = rng.standard_normal((n, H, 2, 64)) * 2.0 ** powers[:, None, :, None]
    moin.kv_append(cache, i32(slot), _dev(k), _dev(ref.bf16(v.reshape(n, H, 128).astype(np.float32))))
    return cache, tables, torch.from_numpy(np.asarray(slot)).to(DEV)


@pytest.mark.parametrize("new,G,n", [(1, 4, 700), (3, 4, 700), (20, 2, 300), (1, 8, 5000)])
@pytest.mark.parametrize("kind", ["first small", "second small", "far apart", "by token", "rising"])
def test_planes_of_a_wide_head_hold_their_own_precision(kind, new, G, n):
    """Value planes 2^30 to 2^90 apart, from the start, token by token, or drifting: each plane is right within bounds of its own size."""
    rng = np.random.default_rng(new + G + len(kind))
    t = np.arange(n)
    powers = {"first small": np.stack([np.full(n, -30.0), np.zeros(n)], -1), "second small": np.stack([np.zeros(n), np.full(n, -45.0)], -1),
              "far apart": np.stack([np.full(n, 45.0), np.full(n, -45.0)], -1), "by token": rng.integers(-25, 26, (n, 2)).astype(float),
              "rising": np.stack([40.0 - 80.0 * t / n, -40.0 + 80.0 * t / n], -1)}[kind]
    H = 2
    cache, tables, slot = _wide(rng, n, H, np.round(powers))
    q = _dev(ref.bf16(rng.standard_normal((new, H * G, 128)).astype(np.float32)))
    pos = torch.arange(n - new, n, device=DEV)
    want, tol = exact.attention(cache, slot, q, pos, 128 ** -0.5, False)
    for max_kv in (n, 0):
        got = moin.kv_attention(cache, tables, q, i32([0, new]), i32([n]), new, max_kv).double()
        assert got.isfinite().all() and ((got - want).abs() <= tol).all(), ((got - want).abs() / tol).max()


@pytest.mark.parametrize("D,H,G,new,n", [(64, 2, 8, 1, 700), (64, 1, 4, 9, 300), (128, 2, 4, 1, 500), (128, 1, 2, 20, 200), (64, 1, 8, 1, 40000)])
@pytest.mark.parametrize("size", [4, 30, 90])
def test_scores_that_jump_by_more_than_fp32_can_add(D, H, G, new, n, size, kernel):
    """Keys of 2^size, of either sign, between ordinary ones: scores rise and fall by 2^size from tile to tile, values' sizes too.  The
    largest keys take all weight, to the last ones of them that a query sees; queries of the other sign see the smallest."""
    if kernel == "tcgen05" and size > 4:
        size -= 20
    rng = np.random.default_rng(size + n + D)
    cache, tables, _, slot = _serve(rng, [n], H, D, 32)
    u = rng.choice([-1.0, 1.0], D)
    a = rng.uniform(-1, 1, n)
    big = rng.permutation(n - new)[:9]
    a[big[:4]], a[big[4:8]] = 2.0 ** size * np.array([1, 1.5, 0.5, 1.25]), -2.0 ** size * np.array([1, 1.5, 0.5, 1.25])
    k = ref.bf16((a[:, None, None] * u).astype(np.float32)) * np.ones((1, H, 1), np.float32)
    v = ref.bf16((rng.standard_normal((n, H, D)) * 2.0 ** rng.integers(-12, 13, (n, 1, 1))).astype(np.float32))
    moin.kv_append(cache, i32(slot), _dev(k), _dev(v))
    sign = np.where(np.arange(new * H * G).reshape(new, H * G) % 2 == 0, 64.0, -64.0)
    q = ref.bf16((sign[..., None] * u).astype(np.float32))
    got = moin.kv_attention(cache, tables, _dev(q), i32([0, new]), i32([n]), new, n).double().cpu().numpy()
    if size == 4:   # ordinary scores: against the formula
        want, tol = exact.attention(cache, torch.from_numpy(np.asarray(slot)).to(DEV), _dev(q), torch.arange(n - new, n, device=DEV), D ** -0.5, kernel == "tcgen05" and D == 64)
        assert (np.abs(got - want.cpu().numpy()) <= tol.cpu().numpy()).all()
        return
    at = np.where(sign > 0, big[1], big[5])
    c, s, z = ref.load(cache.pages.cpu().numpy(), np.asarray(slot), 1)
    val, part = (z[..., None] + s[..., None] * c).reshape(n, H, D), (s[..., None] * c).reshape(n, H, D)
    head = (np.arange(H * G) // G)[None]
    want = val[at, head]
    assert (np.abs(got - want) <= 2.0 ** -8 * np.abs(want) + 2.0 ** -10 * (np.abs(want) + part[at, head]) + 2.0 ** -30 * np.abs(val[at, head]).max(-1, keepdims=True)).all()


def _long(n, H, seed, values, keys=None, page=128):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    pages = -(-n // page)
    cache = moin.KvCache.empty(pages, page, H, 64, DEV)
    slot = torch.arange(n, dtype=torch.int32, device=DEV)
    k = torch.randn(n, H, 64, generator=gen, device=DEV)
    moin.kv_append(cache, slot, (k if keys is None else 0.1 * k + keys).to(torch.bfloat16), values(gen).to(torch.bfloat16))
    tables = moin.KvTables(torch.arange(pages, dtype=torch.int32, device=DEV).view(1, -1), torch.zeros(pages, dtype=torch.int32, device=DEV), page)
    return cache, tables, slot, gen


@pytest.mark.parametrize("n", [65536, 131072, 524288])
def test_long_chunks_hold_their_precision(n):
    """A chunk behind 2^16 to 2^19 tokens, 512 items (more than there are CTAs, so that shares hold whole ones), a flat softmax over
    values with means of their own: sums as long as they get.  Beside the bound: a sum that loses a little the same way at every step
    shows in the mean of the errors along the result, roundings to bf16 do not (they are taken off; what is left of them is 2^-9.3 over the
    root of 6144 results, some of them alike).  2^-12 is a sixteenth of what one rounding may be off by."""
    H, G, m = 4, 8, 2048
    cache, tables, slot, gen = _long(n, H, n, lambda gen: 0.2 * torch.randn(n, H, 64, generator=gen, device=DEV) + (4 + 4 * torch.rand(1, H, 64, generator=gen, device=DEV)) *
                                     torch.where(torch.rand(1, H, 64, generator=gen, device=DEV) < 0.5, -1.0, 1.0))
    q = (0.2 * torch.randn(m, H * G, 64, generator=gen, device=DEV)).to(torch.bfloat16)
    pick = torch.tensor([0, 1000, m - 1], device=DEV)
    moin.set_option(moin.OPT_GEMM_IMPL, 2)
    try:
        got = moin.kv_attention(cache, tables, q, i32([0, m]), i32([n]), m, n)[pick].double()
    finally:
        moin.set_option(moin.OPT_GEMM_IMPL, 0)
    want, tol = exact.attention(cache, slot.long(), q[pick], n - m + pick, 0.125, True)
    assert ((got - want).abs() <= tol).all(), ((got - want).abs() / tol).max()
    drift = ((got - want.to(torch.bfloat16).double()) / want).mean()
    assert drift.abs() <= 2.0 ** -12, drift


@pytest.mark.parametrize("new", [1200, 2400, 5])
@pytest.mark.parametrize("kind", ["rising", "falling", "late"])
def test_long_chunks_whose_maxima_move(kind, new):
    """Scores that rise or fall by 12 over 140 037 tokens, or are all alike but for the last tokens: sums that went to memory meet another
    maximum.  150 items (shares begin inside them), 300, and two."""
    n, H, G = 140037, 2, 8
    t = torch.arange(n, device=DEV)[:, None, None] / n
    u = torch.where(torch.arange(64, device=DEV) % 3 == 0, -1.0, 1.0)
    a = {"rising": 1.5 * t - 0.75, "falling": 0.75 - 1.5 * t, "late": torch.where(t > 0.97, 1.2, -0.3)}[kind]
    cache, tables, slot, gen = _long(n, H, 7, lambda gen: torch.randn(n, H, 64, generator=gen, device=DEV) + 1, a * u)
    q = (u + 0.05 * torch.randn(new, H * G, 64, generator=gen, device=DEV)).to(torch.bfloat16)
    pick = torch.tensor([0, new // 2, new - 1], device=DEV)
    moin.set_option(moin.OPT_GEMM_IMPL, 2)
    try:
        got = moin.kv_attention(cache, tables, q, i32([0, new]), i32([n]), new, n)[pick].double()
    finally:
        moin.set_option(moin.OPT_GEMM_IMPL, 0)
    want, tol = exact.attention(cache, slot.long(), q[pick], n - new + pick, 0.125, True)
    assert ((got - want).abs() <= tol).all(), ((got - want).abs() / tol).max()


@pytest.mark.parametrize("q_scale", [1.0, 8.0, 40.0])
@pytest.mark.parametrize("heads,H", [(16, 2), (4, 4)])
def test_chunks_within_the_bound_of_their_own_formats(heads, H, q_scale):
    """The tensor-core kernel for chunks takes keys and values in fp16: its scores are off by scale 2^-11 sum |q||k| at most, which the
    bound of tests/kv_exact.py has (that of tests/kv_ref.py is for codes as they are); for scores up to several hundred."""
    rng = np.random.default_rng(heads)
    lens, new = [513, 300], [200, 70]
    cache, tables, table, slot = _serve(rng, lens, H, 64, 32)
    q = _dev(ref.bf16((q_scale * rng.standard_normal((270, heads, 64))).astype(np.float32)))
    moin.set_option(moin.OPT_GEMM_IMPL, 2)
    try:
        got = moin.kv_attention(cache, tables, q, i32([0, 200, 270]), i32(lens), 200, 513).double()
    finally:
        moin.set_option(moin.OPT_GEMM_IMPL, 0)
    slot = torch.from_numpy(np.asarray(slot)).to(DEV)
    for a, b, s, n in ((0, 200, slot[:513], 513), (200, 270, slot[513:], 300)):
        want, tol = exact.attention(cache, s, q[a:b], torch.arange(n - (b - a), n, device=DEV), 0.125, True)
        assert ((got[a:b] - want).abs() <= tol).all(), ((got[a:b] - want).abs() / tol).max()
        # the roundings are independent: over 64 products their sum is off by the root of 64 rather than by 64 of them, and the results
        # in the mean square by a sixteenth of the bound and a rounding of their own
        assert (got[a:b] - want).norm() <= (tol / 16 + 2.0 ** -9 * want.abs()).norm()


@pytest.mark.parametrize("D,G,q", [(64, 8, 1), (64, 4, 3), (64, 4, 30), (128, 4, 1), (128, 4, 3), (128, 2, 20)])
@pytest.mark.parametrize("kind", ["one", "few", "many short", "more than there are CTAs"])
def test_attention_under_loose_bounds(kind, D, G, q):
    """Short requests that were declared as long as their rows, and rows that hold much more: most shares are empty, and requests
    without queries or tokens stand between the others."""
    rng = np.random.default_rng(D + G + q + len(kind))
    lens = {"one": [37], "few": [31, 0, 5, 60, 17], "many short": [int(x) for x in rng.integers(0, 60, 40)],
            "more than there are CTAs": [int(x) for x in rng.integers(0, 40, 300)]}[kind]
    H = 4 if kind == "more than there are CTAs" else 2
    if kind == "more than there are CTAs" and q > 1:
        lens = lens[:110]
    new = [0 if i % 5 == 3 else min(q, n) if n else i % 2 for i, n in enumerate(lens)]
    cache, tables, table, _ = _serve(rng, lens, H, D, 32)
    wide = np.full((len(lens), 300), -1, np.int64)      # rows of 9600 tokens
    wide[:, :table.shape[1]] = table
    tables = moin.KvTables(i32(wide), torch.zeros(cache.n_pages, dtype=torch.int32, device=DEV), 32)
    cu = np.concatenate([[0], np.cumsum(new)])
    T = int(cu[-1])
    x = ref.bf16(rng.standard_normal((T + 2, H * G, D)).astype(np.float32))
    want, tol = ref.attention(cache.pages.cpu().numpy(), wide, None, cu, lens, x, D ** -0.5, 32)
    moin.set_option(moin.OPT_GEMM_IMPL, 1)
    try:
        for max_q in (0, max(q, 1)):
            out = torch.full((T + 2, H * G, D), 9.0, dtype=torch.bfloat16, device=DEV)
            moin.kv_attention(cache, tables, _dev(x), i32(cu), i32(lens), max_q, 0, out=out)
            got = out.double().cpu().numpy()
            assert (got[T:] == 9).all()
            assert (np.abs(got[:T] - want[:T]) <= tol[:T]).all(), np.nanmax(np.abs(got[:T] - want[:T]))
    finally:
        moin.set_option(moin.OPT_GEMM_IMPL, 0)


@pytest.mark.parametrize("D,H,G,new,n", [(64, 2, 8, 1, 700), (64, 1, 4, 70, 300), (128, 2, 4, 1, 500), (128, 1, 2, 20, 200), (64, 1, 8, 1, 40000)])
@pytest.mark.parametrize("size", [10, 16, 24, 40])
def test_scores_that_are_all_far_below_zero(D, H, G, new, n, size, kernel):
    """Every score is between -2^size and -2^(size + 1) times 64 or so; the least negative key, seen by all, takes all weight: the next one is
    2^-5 of its size further, hundreds and more in the exponent."""
    rng = np.random.default_rng(size + n)
    cache, tables, _, slot = _serve(rng, [n], H, D, 32)
    u = rng.choice([-1.0, 1.0], D)
    a = -rng.uniform(1.0625, 2, n)
    best = int(rng.integers(0, n - new + 1))
    a[best] = -1
    k = ref.bf16((2.0 ** size * a[:, None, None] * u).astype(np.float32)) * np.ones((1, H, 1), np.float32)
    v = ref.bf16((rng.standard_normal((n, H, D)) * 2.0 ** rng.integers(-12, 13, (n, 1, 1))).astype(np.float32))
    moin.kv_append(cache, i32(slot), _dev(k), _dev(v))
    q = ref.bf16(np.broadcast_to(64 * u, (new, H * G, D)).astype(np.float32))
    got = moin.kv_attention(cache, tables, _dev(q), i32([0, new]), i32([n]), new, n).double().cpu().numpy()
    c, s, z = ref.load(cache.pages.cpu().numpy(), np.asarray(slot)[best:best + 1], 1)
    head = np.arange(H * G) // G
    val, part = ((z[..., None] + s[..., None] * c).reshape(H, D)[head], (s[..., None] * c).reshape(H, D)[head])
    assert (np.abs(got - val) <= 2.0 ** -8 * np.abs(val) + 2.0 ** -10 * (np.abs(val) + part) + 2.0 ** -30 * np.abs(val).max(-1, keepdims=True)).all()


@pytest.mark.parametrize("D,H,G,new,n", [(64, 2, 8, 1, 700), (64, 1, 4, 70, 400), (128, 2, 4, 1, 500), (128, 1, 2, 20, 300), (64, 1, 8, 1, 40000), (128, 1, 7, 48, 6000)])
@pytest.mark.parametrize("size", [18, 24, 40, 80])
@pytest.mark.parametrize("values", [-40, 0, 47])
def test_scores_that_come_back_from_far_below_zero(D, H, G, new, n, size, values, kernel):
    """Keys of -2^size and less, then ordinary ones: the first leave no weight, the rest is the formula over the others; values of any
    size, planes of a wide head of their own."""
    rng = np.random.default_rng(size + n + values)
    cache, tables, _, slot = _serve(rng, [n], H, D, 32)
    u, half = rng.choice([-1.0, 1.0], D), n // 2
    a = np.concatenate([-2.0 ** size * rng.uniform(1, 2, half), np.zeros(n - half)])
    k = a[:, None, None] * u + np.where(np.arange(n) < half, 0, 1)[:, None, None] * rng.standard_normal((n, H, D))
    v = rng.standard_normal((n, H, D // 64, 64)) * 2.0 ** (values + 12 * rng.uniform(-1, 1, (n, 1, D // 64, 1)))
    moin.kv_append(cache, i32(slot), _dev(ref.bf16(k.astype(np.float32))), _dev(ref.bf16(v.reshape(n, H, D).astype(np.float32))))
    q = _dev(ref.bf16((4 * u + rng.standard_normal((new, H * G, D))).astype(np.float32)))
    got = moin.kv_attention(cache, tables, q, i32([0, new]), i32([n]), new, n).double()
    slot = torch.from_numpy(np.asarray(slot)).to(DEV)[half:]
    want, tol = exact.attention(cache, slot, q, torch.arange(n - new, n, device=DEV) - half, D ** -0.5, kernel == "tcgen05" and D == 64)
    assert got.isfinite().all() and ((got - want).abs() <= tol).all(), ((got - want).abs() / tol).max()
