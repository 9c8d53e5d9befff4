"""Results of cached attention in the memory of its queries: refused where they overlap (a request's CTAs read queries while others
write results), taken where they lie side by side in the rows of one tensor."""
import numpy as np
import pytest
import torch

import kv_ref as ref
import paper_2410_09687_b200 as moin
from test_gpu_kv import DEV, _dev, _serve, i32

pytestmark = pytest.mark.gpu


def test_overlap():
    rng = np.random.default_rng(1)
    lens, heads, D = [300, 40, 7], 4, 64
    cache, tables, _, _ = _serve(rng, lens, 2, D, 16)
    T, W = 6, heads * D
    x = _dev(ref.bf16(rng.standard_normal((T, heads, D)).astype(np.float32)))
    args = (i32([0, 3, 5, 6]), i32(lens), 3, 300)
    want = moin.kv_attention(cache, tables, x, *args)
    wide = torch.zeros(T, 3 * W, dtype=torch.bfloat16, device=DEV)
    part = lambda at: wide[:, at:at + W].view(T, heads, D)  # noqa: E731
    part(W).copy_(x)
    for at in (0, 2 * W):                                   # beside the queries
        out = moin.kv_attention(cache, tables, part(W), *args, out=part(at))
        assert torch.equal(out, want) and torch.equal(part(W), x)
    flat = torch.zeros(3 * T, heads, D, dtype=torch.bfloat16, device=DEV)
    flat[T:2 * T] = x
    for a in (0, 2 * T):                                    # behind and before them
        assert torch.equal(moin.kv_attention(cache, tables, flat[T:2 * T], *args, out=flat[a:a + T]), want)
    for q, out in ((x, x), (part(W), part(W)), (part(W), part(W + 8)), (part(W), part(W - 8)), (part(0), part(W - D)), (flat[T:2 * T], flat[2 * T - 1:3 * T - 1]),
                   (flat[T:2 * T], flat[1:1 + T]), (flat[:T], flat[::2][:T]), (part(0), wide.view(-1)[:T * W].view(T, heads, D))):
        before = out.clone()
        with pytest.raises(moin.MoinError, match="overlap"):
            moin.kv_attention(cache, tables, q, *args, out=out)
        assert torch.equal(out, before)
