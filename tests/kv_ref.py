"""Plain restatements of the 4-bit key/value cache in numpy, written from the format and formulas of include/moin.h: byte
layout looked up entry by entry, tables by a walk over the requests, attention in fp64."""
import numpy as np
import torch

TILE_BYTES = 1152


def bf16(x):
    return torch.from_numpy(np.ascontiguousarray(x)).to(torch.bfloat16).float().numpy()


def quantise(x):
    """x [..., 64] float32 (bf16 values) -> codes, scale [...], zero [...]."""
    x = np.asarray(x, np.float32)
    lo, hi = x.min(-1), x.max(-1)
    with np.errstate(over="ignore", invalid="ignore"):
        span = (hi - lo).astype(np.float32)
        scale = bf16(np.maximum(np.maximum(span / np.float32(15), np.abs(lo) * np.float32(2.0 ** -12)), np.float32(2.0 ** -64)))
        bad = ~np.isfinite(x).all(-1) | ~np.isfinite(span)
        code = np.clip(np.rint((x - lo[..., None]) / scale[..., None]), 0, 15)
    code = np.where(bad[..., None], 0, code).astype(np.int64)
    return code, np.where(bad, np.nan, scale), np.where(bad, np.nan, lo)


def values(x):
    """What a row stands for once stored, in fp64."""
    c, s, z = quantise(x)
    return z.astype(np.float64)[..., None] + s.astype(np.float64)[..., None] * c


def rotate(x, pos, table):
    """x [T, heads, D] float32, table [n, D/2, 2] float32: every operation rounded to fp32, the result to bf16."""
    cs = table[pos][:, None]
    h = x.shape[-1] // 2
    a, b, c, s = x[..., :h], x[..., h:], cs[..., 0], cs[..., 1]
    return bf16(np.concatenate([a * c - b * s, b * c + a * s], -1).astype(np.float32))


def byte_of(kv, tok, ch):
    """(byte of a tile, 0 = low or 4 = high half) of a token's channel; kv 0 = key, 1 = value."""
    j, half, r = ch // 16, ch // 8 % 2, ch % 8
    if kv == 0:
        s, g, t, c = tok // 8, tok % 8, r // 2, r % 2
    else:
        s, t, c, g = tok // 8, tok % 8 // 2, tok % 2, r
    return 512 * kv + (((g * 4 + t) * 4 + j) * 2 + c) * 2 + s, 4 * half


def pair_of(kv, tok):
    return 1024 + ((tok % 8) * 2 + kv) * 8 + (tok // 8) * 4


def store(pages, slot, x, kv):
    """Writes rows x [T, H, D] (float32 holding bf16 values) into the byte array pages [n, H, tiles, planes, 1152]."""
    n, H, tiles, planes, _ = pages.shape
    P = tiles * 16
    code, scale, zero = quantise(np.asarray(x, np.float32).reshape(len(slot), H, planes, 64))
    for t, s in enumerate(slot):
        if s < 0 or s >= n * P:
            continue
        page, tile, tok = s // P, s % P // 16, s % 16
        for h in range(H):
            for p in range(planes):
                row = pages[page, h, tile, p]
                for ch in range(64):
                    b, sh = byte_of(kv, tok, ch)
                    row[b] = (row[b] & (0xF0 >> sh)) | (code[t, h, p, ch] << sh)
                two = torch.tensor([scale[t, h, p], zero[t, h, p]], dtype=torch.float32).to(torch.bfloat16).view(torch.uint8).numpy()
                row[pair_of(kv, tok):pair_of(kv, tok) + 4] = two


def load(pages, slot, kv, dtype=np.float64):
    """(codes, scale, zero) of slots as arrays [T, H, planes, 64], [T, H, planes]."""
    n, H, tiles, planes, _ = pages.shape
    P = tiles * 16
    slot = np.asarray(slot)
    where = [[byte_of(kv, tok, ch) for ch in range(64)] for tok in range(16)]
    byte = np.array([[w[0] for w in r] for r in where])[slot % 16]
    shift = np.array([[w[1] for w in r] for r in where])[slot % 16]
    tiles_of = pages[slot // P, :, slot % P // 16]                                   # T, H, planes, 1152
    code = (np.take_along_axis(tiles_of, np.broadcast_to(byte[:, None, None], tiles_of.shape[:3] + (64,)), -1) >> shift[:, None, None]) & 15
    at = np.array([pair_of(kv, tok) for tok in range(16)])[slot % 16][:, None, None, None] + np.arange(4)
    raw = np.take_along_axis(tiles_of, np.broadcast_to(at, tiles_of.shape[:3] + (4,)), -1).astype(np.uint32)
    word = lambda i: ((raw[..., i] | raw[..., i + 1] << 8) << 16).astype(np.uint32).view(np.float32).astype(dtype)  # noqa: E731
    return code.astype(dtype), word(0), word(2)


def update(table, stack, lens, n_free, want, rows, page, T):
    """moin_kv_update, request by request."""
    table, stack, lens = table.copy(), stack.copy(), lens.copy()
    n_rows, max_pages = table.shape
    R, pages = len(want), lambda n: -(-n // page)
    rows = np.arange(R) if rows is None else rows
    named = [0 <= r < n_rows and list(rows).count(r) == 1 for r in rows]
    good = [n and 0 <= lens[r] <= max_pages * page and 0 <= w <= max_pages * page for n, r, w in zip(named, rows, want)]
    for g, r, w in zip(good, rows, want):
        if g:
            for p in range(pages(int(w)), pages(int(lens[r]))):
                stack[n_free] = table[r, p]
                n_free += 1
    top, taken, asked, refused = n_free, 0, 0, 0
    cu, kv, slot, pos = [0], [], np.full(T, -1, np.int64), np.full(T, -1, np.int64)
    tokens = 0
    for g, r, w in zip(good, rows, want):
        if not g:
            refused += 1
            cu.append(min(tokens, T))
            kv.append(0)
            continue
        w, old = int(w), int(lens[r])
        new, first = max(0, w - old), tokens
        tokens += new
        cu.append(min(tokens, T))
        ok = new == 0 or tokens <= T
        if ok:
            ask = max(0, pages(w) - pages(old))
            asked += ask
            ok = ask == 0 or asked <= top
        if not ok:
            refused += 1
            kv.append(0)
            continue
        for p in range(pages(old), pages(w)):
            table[r, p] = stack[top - 1 - taken]
            taken += 1
        for i in range(new):
            pos[first + i] = old + i
            slot[first + i] = table[r, (old + i) // page] * page + (old + i) % page
        kv.append(w)
        lens[r] = w
    return {"block_table": table, "free_pages": stack, "lens": lens, "n_free": np.array([top - taken]), "refused": np.array([refused]),
            "cu_q": np.array(cu), "kv_len": np.array(kv), "slot": slot, "pos": pos}


def attention(pages, table, rows, cu_q, kv_len, q, scale, page):
    """q [T, heads, D] float32 (rotated already) -> out [T, heads, D] and a bound on the error of a computation that rounds the
    weights p sv to fp16 and the result to bf16 and does the rest in fp32:
      2^-8 |o|                           the result (half a bf16 step)
      2^-11 sum p (sv c) / sum p         the weights (half an fp16 step, relative)
      (2^-17 B + 2^-18) max |v|          scores: products are exact, the sums of 64 to 128 of them err by at most 2^-19 B in a
                                         tensor-core accumulator, B = scale sum |q| max(|zk| + 15 sk); a relative error d of the
                                         weights moves o by at most 2 d max |v| (and twice that for both of sum p v and sum p);
                                         2^-18: exponentials, and sums over tokens in fp32 (up to 4096 of them)."""
    H = pages.shape[1]
    T, heads, D = q.shape
    G = heads // H
    out, tol = np.full((T, heads, D), np.nan), np.zeros((T, heads, D))
    for i in range(len(kv_len)):
        t0, t1, n = int(cu_q[i]), int(cu_q[i + 1]), int(kv_len[i])
        if t1 == t0:
            continue
        row = i if rows is None else int(rows[i])
        where = np.arange(n)
        page_of = table[row, where // page] if n else np.zeros(0, np.int64)
        there = (page_of >= 0) & (page_of < pages.shape[0])
        slot = np.where(there, page_of, 0) * page + where % page
        out[t0:t1] = 0
        if not n:
            continue
        kc, ks, kz = load(pages, slot, 0)
        vc, vs, vz = load(pages, slot, 1)
        K = (kz[..., None] + ks[..., None] * kc).reshape(n, H, D)
        V = (vz[..., None] + vs[..., None] * vc).reshape(n, H, D)
        for j in range(t0, t1):
            seen = np.nonzero(there & (where <= n - (t1 - t0) + (j - t0)))[0]
            if not len(seen):
                continue
            for h in range(heads):
                kv = h // G
                qr = q[j, h].astype(np.float64)
                s = scale * (K[seen, kv] @ qr)
                p = np.exp(s - s.max())
                p /= p.sum()
                o = p @ V[seen, kv]
                B = abs(scale) * np.abs(qr).sum() * (np.abs(kz[seen, kv]) + 15 * ks[seen, kv]).max()
                A = (p @ (vs[seen, kv][..., None] * vc[seen, kv]).reshape(len(seen), D))
                out[j, h] = o
                tol[j, h] = 2.0 ** -8 * np.abs(o) + 2.0 ** -11 * A + (2.0 ** -17 * B + 2.0 ** -18) * np.abs(V[seen, kv]).max()
    return out, tol
