"""Attention over the 4-bit cache in fp64 on the GPU, for requests too long for tests/kv_ref.py, with a bound on the error that is
written for each kernel and for each plane of 64 channels by itself."""
import torch

import kv_ref as ref


def stored(cache, kv):
    """(codes [slots, H, planes, 64], scale, zero [slots, H, planes]) of a whole cache, from the byte layout of include/moin.h."""
    pages = cache.pages
    n, H, tiles, planes, _ = pages.shape
    where = torch.tensor([[ref.byte_of(kv, tok, ch) for ch in range(64)] for tok in range(16)], device=pages.device)
    at = torch.tensor([ref.pair_of(kv, tok) for tok in range(16)], device=pages.device)
    code = (pages[..., where[..., 0]] >> where[..., 1].to(torch.uint8)) & 15
    pair = pages[..., at[:, None] + torch.arange(4, device=pages.device)].contiguous().view(torch.bfloat16)
    code = code.permute(0, 2, 4, 1, 3, 5).reshape(n * tiles * 16, H, planes, 64)
    pair = pair.permute(0, 2, 4, 1, 3, 5).reshape(n * tiles * 16, H, planes, 2).double()
    return code, pair[..., 0], pair[..., 1]


def attention(cache, slots, q, pos, scale, chunk):
    """q [m, heads, D] (rotated) at positions pos [m] of the request whose token t is in slots[t] -> (out [m, heads, D], tol), fp64.
    With p the weights of the softmax, v = z + s c a value, in a plane with max |v| = M over the tokens seen, n tokens:
      2^-8 |o|                        the result, half a bf16 step
      expm1(2 d) M                    scores that are off by d each move o by no more.  d = 2^-18 B + 2^-19: B = scale sum|q| max|k|, products
                                      are exact and the sums of 64 to 128 of them err by at most 2^-19 B on a tensor core, as much again
                                      for scale and zero applied in fp32; 2^-19 for the exponential
    chunk = False (codes as they are):
      2^-11 sum p s c                 weights rounded to fp16, half a step
      15 n 2^-35 sum p s              weights below 2^-14 are off by 2^-25, where the plane's largest is 2^10 at least
      n 2^-28 sum p (|z| + 15 s)      fp32 sums over n / 16 tiles
    chunk = True (keys and values in fp16, a tile's largest at 2^13 and more):
      d grows by 2^-11 scale sum |q||k|    half a step of the keys
      2 2^-11 sum p |v| + 2^-30 M          half a step of values and weights; what is lost below fp16's least normal value
      n 2^-29 max p M                      weights below 2^-14, off by 2^-25, where the row's largest is 2^5 at least
      n 2^-25 sum p |v|                    fp32 sums over the tiles and inside the tensor core"""
    m, heads, D = q.shape
    H, planes = cache.n_kv_heads, D // 64
    G, n_all = heads // H, len(slots)
    code = {kv: [x[slots] for x in stored(cache, kv)] for kv in range(2)}
    out, tol = (torch.zeros(m, heads, planes, 64, dtype=torch.float64, device=q.device) for _ in range(2))
    seen = torch.arange(n_all, device=q.device) <= pos[:, None]
    n = seen.sum(-1)[:, None, None].double()
    for h in range(H):
        (kc, ks, kz), (vc, vs, vz) = ([x[:, h].double() for x in code[kv]] for kv in range(2))
        K = (kz[..., None] + ks[..., None] * kc).reshape(n_all, D)
        for g in range(h * G, (h + 1) * G):
            x = q[:, g].double()
            s = (scale * (x @ K.T)).masked_fill(~seen, float("-inf"))
            p = torch.softmax(s, -1)
            B = abs(scale) * x.abs().sum(-1) * K.abs().max()
            d = 2.0 ** -18 * B + 2.0 ** -19
            if chunk:
                d = d + 2.0 ** -11 * abs(scale) * (x.abs() @ K.abs().T).masked_fill(~seen, 0.0).amax(-1)
            for pl in range(planes):
                V = vz[:, pl, None] + vs[:, pl, None] * vc[:, pl]
                o = p @ V
                M = V.abs().amax(-1).expand(m, -1).masked_fill(~seen, 0.0).amax(-1)
                t = 2.0 ** -8 * o.abs() + torch.expm1(2 * d).clamp(max=2.0)[:, None] * M[:, None]
                if chunk:
                    V = V.abs()
                    t = t + (2.0 ** -10 + n[:, 0] * 2.0 ** -25) * (p @ V) + (2.0 ** -30 + n[:, 0] * 2.0 ** -29 * p.amax(-1, keepdim=True)) * M[:, None]
                else:
                    t = t + 2.0 ** -11 * (p @ (vs[:, pl, None] * vc[:, pl])) + n[:, 0] * (15 * 2.0 ** -35 * (p @ vs[:, pl])[:, None] + 2.0 ** -28 * (p @ (vz[:, pl].abs() + 15 * vs[:, pl]))[:, None])
                out[:, g, pl], tol[:, g, pl] = o, t
    return out.view(m, heads, D), tol.view(m, heads, D)
