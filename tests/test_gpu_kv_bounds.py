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
