"""What serving from a 4-bit key/value cache costs, operator by operator.

Three kinds of work, as a server that generates text does them every step:

  tables     wanted request lengths -> pages taken and given back, slot and position of every new token (``kv_update``)
  append     new keys and values -> rotated, quantised to 4 bits and stored by slot (``kv_append``), and the stored rows
             read back as the values they stand for (``kv_read``)
  attention  queries over a request's cached tokens (``kv_attention``): one token a request, a few, or a prompt's chunk

`run` computes them in plain torch operations in 32 bits, or (`own`) by this repository's entry points.

The cache is a byte tensor [pages, kv heads, 16-token tiles of a page, 64-channel planes, 1152].  The 64 channels of a
token's key (or value) in a plane are a row: its smallest value `zero` and a step `scale` (both bf16) and 64 codes of 4
bits, value = zero + scale * code.  The 1152 bytes of a tile are 512 of keys, 512 of values, 128 of (scale, zero) pairs:
  keys    byte (g, t, j, c, s) in mixed radix 8, 4, 4, 2, 2 holds token 8 s + g; channel 16 j + 2 t + c in its low half, 8 more in its high half
  values  byte (g, t, j, c, s) holds token 8 s + 2 t + c; channel 16 j + g in its low half, 8 more in its high half
  pairs   32-bit word (g, kv, s) of token 8 s + g: scale in the low half, zero in the high half; kv 0 = key, 1 = value
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda"
TILE = 16            # tokens of a tile
TILE_BYTES = 1152


def listed():
    return [
        # the table of a server with one running request that takes one more token
        {"name": "tables_one", "kind": "tables", "R": 1, "rows": 8, "page": 16, "lo": 700, "hi": 700, "new_lo": 1, "new_hi": 1,
         "done": 0.0, "spare": 64},
        # a decode step of a busy server: one token each, some requests done and their pages back
        {"name": "tables_decode_256", "kind": "tables", "R": 256, "rows": 512, "page": 64, "lo": 16, "hi": 8192, "new_lo": 1,
         "new_hi": 1, "done": 0.06, "spare": 4096},
        # prompts enter, more of them than there are free pages
        {"name": "tables_prompts", "kind": "tables", "R": 97, "rows": 128, "page": 16, "lo": 1, "hi": 512, "new_lo": 33,
         "new_hi": 2048, "done": 0.1, "spare": 3000},
        # one token of one request (heads of the 1.1B model: 4 key/value heads of 64)
        {"name": "append_one", "kind": "append", "R": 1, "H": 4, "D": 64, "page": 16, "lo": 900, "hi": 900, "new_lo": 1, "new_hi": 1},
        # a decode step: a token each, every one in a page of its own
        {"name": "append_decode_256", "kind": "append", "R": 256, "H": 4, "D": 64, "page": 64, "lo": 16, "hi": 8192,
         "new_lo": 1, "new_hi": 1},
        # ragged prompts behind ragged pasts, wider heads
        {"name": "append_prompts", "kind": "append", "R": 37, "H": 8, "D": 128, "page": 32, "lo": 1, "hi": 700,
         "new_lo": 65, "new_hi": 2048},
        # the smallest call: one short request generates a token
        {"name": "decode_one_short", "kind": "attention", "R": 1, "heads": 32, "H": 4, "D": 64, "page": 16, "lo": 193, "hi": 193,
         "new_lo": 1, "new_hi": 1},
        # one request at the end of a long document
        {"name": "decode_one_long", "kind": "attention", "R": 1, "heads": 32, "H": 4, "D": 64, "page": 64, "lo": 131071, "hi": 131071,
         "new_lo": 1, "new_hi": 1},
        # a decode step of a busy server, lengths spread over a factor of sixteen
        {"name": "decode_256", "kind": "attention", "R": 256, "heads": 32, "H": 4, "D": 64, "page": 64, "lo": 512, "hi": 8192,
         "new_lo": 1, "new_hi": 1},
        # the same with heads of 128 in groups of four, small pages
        {"name": "decode_64_wide", "kind": "attention", "R": 64, "heads": 32, "H": 8, "D": 128, "page": 16, "lo": 256, "hi": 8191,
         "new_lo": 1, "new_hi": 1},
        # several guessed tokens a request checked at once
        {"name": "verify_48", "kind": "attention", "R": 48, "heads": 32, "H": 4, "D": 64, "page": 32, "lo": 129, "hi": 6000,
         "new_lo": 2, "new_hi": 8},
        # chunks of long prompts behind what is cached of them
        {"name": "chunk_4x512", "kind": "attention", "R": 4, "heads": 32, "H": 4, "D": 64, "page": 64, "lo": 600, "hi": 8192,
         "new_lo": 512, "new_hi": 512},
    ]


def _log(rng, lo, hi):
    return int(round(lo * (hi / lo) ** rng.random()))


def draw(rng):
    """Cases of the listed ranges: tokens, requests and cached lengths spread over their logarithm."""
    kind = rng.choice(["tables", "append", "attention", "attention"])
    page = rng.choice([16, 32, 64, 128])
    if kind == "tables":
        R = _log(rng, 1, 512)
        prompts = rng.random() < 0.5 and R <= 128
        new_hi = _log(rng, 2, 1024) if prompts else 1
        return {"kind": kind, "R": R, "rows": R + rng.randint(0, 64), "page": page, "lo": rng.randint(1, 64),
                "hi": _log(rng, 64, 4096), "new_lo": rng.randint(1, new_hi), "new_hi": new_hi, "done": rng.choice([0.0, 0.1, 0.3]),
                "spare": _log(rng, 16, 4096)}
    H, D = rng.choice([1, 2, 4, 8]), rng.choice([64, 64, 128])
    if kind == "append":
        R = _log(rng, 1, 256)
        new_hi = rng.choice([1, _log(rng, 2, max(3, min(2048, 16384 // R)))])
        return {"kind": kind, "R": R, "H": H, "D": D, "page": page, "lo": rng.randint(1, 300), "hi": _log(rng, 300, 4000),
                "new_lo": rng.randint(1, new_hi), "new_hi": new_hi}
    heads = H * rng.choice([1, 2, 4, 7, 8, 16])
    hi = _log(rng, 40, 32768)
    most = max(1, min(256, 2 ** 26 // (hi * H * D)))     # what the plain form unpacks of each of keys and values
    R = _log(rng, 1, most)
    longest = max(1, min(hi, 400, 2 ** 26 // (R * hi * heads)))
    new_hi = rng.choice([1, 1, rng.randint(1, min(8, longest)), _log(rng, 1, longest)])
    return {"kind": kind, "R": R, "heads": heads, "H": H, "D": D, "page": page, "lo": rng.randint(1, 40), "hi": hi,
            "new_lo": rng.randint(1, new_hi), "new_hi": new_hi}


def _spread(lo, hi, n):
    """n lengths from lo to hi, evenly spread over their logarithm: the same for every seed, so that the work is the case's."""
    at = (np.arange(n) + 0.5) / max(n, 1)
    return np.clip(np.round(lo * (hi / lo) ** at), lo, hi).astype(np.int64)


def _lengths(case):
    """Cached tokens before the call and new tokens, request by request (request order is drawn in prepare)."""
    old = _spread(case["lo"], case["hi"], case["R"])
    new = _spread(case["new_lo"], case["new_hi"], case["R"])
    new = new[(np.arange(case["R"]) * 7919 + 13) % case["R"]] if case["R"] % 7919 else new
    return old, new


def _pages(tokens, page):
    return (tokens + page - 1) // page


def prepare(case, seed):
    rng = np.random.default_rng([seed, 4])
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    R, page = case["R"], case["page"]
    old, new = _lengths(case)
    done = np.arange(R) * 7 % R < int(case.get("done", 0.0) * R) if R % 7 else np.arange(R) < int(case.get("done", 0.0) * R)
    order = rng.permutation(R)
    old, new, done = old[order], new[order], done[order]
    i32 = lambda a: torch.from_numpy(np.ascontiguousarray(a, np.int32)).to(DEV)  # noqa: E731
    state = {"case": case}
    if case["kind"] == "tables":
        n_rows = case["rows"]
        others = rng.permutation(n_rows)
        rows, others = others[:R], others[R:]
        lens = np.zeros(n_rows, np.int64)
        lens[rows], lens[others] = old, _spread(case["lo"], case["hi"], n_rows - R)
        want = np.where(done, 0, old + new)
        have = _pages(lens, page)
        max_pages = int(max(have.max(), _pages(want, page).max()))
        n_pages = int(have.sum()) + case["spare"]
        ids = rng.permutation(n_pages)
        table = np.zeros((n_rows, max_pages), np.int32)
        table[np.arange(max_pages) < have[:, None]] = ids[:have.sum()]
        free = np.zeros(n_pages, np.int32)
        free[:case["spare"]] = ids[have.sum():]
        T = int(np.where(done, 0, new).sum())
        state |= {"rows": i32(rows), "want": i32(want), "lens": i32(lens), "n_free": i32([case["spare"]]), "block_table": i32(table),
                  "free_pages": i32(free), "T": T, "lens_out": i32(lens), "n_free_out": i32([0])}
        if own:   # the structs over these buffers that a server keeps
            import paper_2410_09687_b200 as moin
            state["tables"] = moin.KvTables(state["block_table"], state["free_pages"], page, state["lens"], state["n_free"])
            state["batch"] = moin.KvBatch(R, T, DEV)
        return state

    H, D = case["H"], case["D"]
    total = old + new
    have = _pages(total, page)
    n_pages = int(have.sum()) + 3
    max_pages = int(have.max())
    ids = rng.permutation(n_pages)
    table = np.zeros((R, max_pages), np.int32)
    table[np.arange(max_pages) < have[:, None]] = ids[:have.sum()]
    cu = np.concatenate([[0], np.cumsum(new)])
    T = int(cu[-1])
    at = np.arange(T) - np.repeat(cu[:-1], new)
    pos = np.repeat(old, new) + at
    req = np.repeat(np.arange(R), new)
    slot = table[req, pos // page].astype(np.int64) * page + pos % page
    angle = np.arange(max_pages * page)[:, None] * 10000.0 ** (-np.arange(D // 2) / (D // 2))
    rope = torch.from_numpy(np.stack([np.cos(angle), np.sin(angle)], -1).astype(np.float32)).to(DEV)
    state |= {"rope": rope, "slot": i32(slot), "pos": i32(pos), "T": T}
    # keys have a few channels that stand out and a mean of their own, values do not
    wide = torch.ones(H, D, device=DEV)
    wide[:, torch.randperm(D, generator=gen, device=DEV)[:D // 16]] = 3.0
    mean = 0.5 * torch.randn(H, D, generator=gen, device=DEV) * wide
    shape = (n_pages, H, page // TILE, D // 64, TILE_BYTES)
    if case["kind"] == "append":
        state["k"] = (torch.randn(T, H, D, generator=gen, device=DEV) * wide + mean).to(torch.bfloat16)
        state["v"] = torch.randn(T, H, D, generator=gen, device=DEV).to(torch.bfloat16)
        state["pages"] = torch.zeros(shape, dtype=torch.uint8, device=DEV)
    else:
        pages = torch.empty(shape, dtype=torch.uint8, device=DEV)
        for p0 in range(0, n_pages, max(1, 2 ** 25 // (page * H * D))):     # a piece of the cache at a time
            n = min(n_pages - p0, max(1, 2 ** 25 // (page * H * D)))
            k = (torch.randn(n, page, H, D, generator=gen, device=DEV) * wide + mean).to(torch.bfloat16).float()
            v = torch.randn(n, page, H, D, generator=gen, device=DEV).to(torch.bfloat16).float()
            pages[p0:p0 + n] = _pack(*_quantise(k), *_quantise(v))
        state["pages"] = pages
        state["q"] = (1.5 * torch.randn(T, case["heads"], D, generator=gen, device=DEV)).to(torch.bfloat16)
        state["block_table"] = i32(table)
        state["cu_q"], state["kv_len"] = i32(cu), i32(total)
        state["max_q"], state["max_kv"] = int(new.max()), int(total.max())
    if own:
        import paper_2410_09687_b200 as moin
        state["cache"] = moin.KvCache(state["pages"])
        if case["kind"] == "attention":
            state["tables"] = moin.KvTables(state["block_table"], torch.zeros(n_pages, dtype=torch.int32, device=DEV), page)
    return state


# ------------------------------------------------------------------------------------------------ the format, plain
def _quantise(x):
    """x [..., D] float32 holding bf16 values -> codes [..., D/64, 64] uint8, scale and zero [..., D/64] (bf16 values as float32)."""
    x = x.reshape(*x.shape[:-1], -1, 64)
    lo, hi = x.amin(-1), x.amax(-1)
    step = (hi - lo) / torch.full_like(lo, 15.0)      # (by a tensor: torch multiplies by the inverse of a plain number)
    scale = torch.maximum(torch.maximum(step, lo.abs() * 2.0 ** -12), torch.full_like(lo, 2.0 ** -64)).to(torch.bfloat16).float()
    code = torch.round((x - lo[..., None]) / scale[..., None]).clamp(0, 15)
    return code.to(torch.uint8), scale, lo


def _pack(kc, ks, kz, vc, vs, vz):
    """Codes [pages, page, H, planes, 64] and their pairs -> bytes [pages, H, tiles, planes, 1152]."""
    n, page, H, P, _ = kc.shape
    t = page // TILE
    # keys: token (s, g), channel (j, half, t, c) -> byte (g, t, j, c, s)
    k = kc.reshape(n, t, 2, 8, H, P, 4, 2, 4, 2).permute(0, 4, 1, 5, 3, 8, 6, 9, 2, 7)
    # values: token (s, t, c), channel (j, half, g) -> byte (g, t, j, c, s)
    v = vc.reshape(n, t, 2, 4, 2, H, P, 4, 2, 8).permute(0, 5, 1, 6, 9, 3, 7, 4, 2, 8)
    both = [(x[..., 0] | (x[..., 1] << 4)).reshape(n, H, t, P, 512) for x in (k, v)]
    pairs = torch.stack([torch.stack([s, z], -1) for s, z in ((ks, kz), (vs, vz))], -2).to(torch.bfloat16)   # [n, page, H, P, kv, 2]
    pairs = pairs.reshape(n, t, 2, 8, H, P, 2, 2).permute(0, 4, 1, 5, 3, 6, 2, 7).contiguous()
    return torch.cat(both + [pairs.view(torch.uint8).reshape(n, H, t, P, 128)], -1)


def _unpack(b, kind=torch.float32):
    """Bytes [..., H, tiles, planes, 1152] -> keys and values [..., H, tiles * 16, planes * 64]."""
    lead, (H, t, P, _) = b.shape[:-4], b.shape[-4:]
    pairs = b[..., 1024:].contiguous().view(torch.bfloat16).reshape(-1, H, t, P, 8, 2, 2, 2).to(kind)   # g, kv, s, (scale, zero)
    out = []
    for kv in range(2):
        c = b[..., 512 * kv:512 * (kv + 1)].reshape(-1, H, t, P, 8, 4, 4, 2, 2)
        c = torch.stack([c & 15, c >> 4], -1)                                    # n, H, t, P, g, t, j, c, s, half
        c = c.permute(0, 1, 2, 8, 4, 3, 6, 9, 5, 7) if kv == 0 else c.permute(0, 1, 2, 8, 5, 7, 3, 6, 9, 4)
        c = c.reshape(-1, H, t * TILE, P, 64).to(kind)
        sz = pairs[..., kv, :, :].permute(0, 1, 2, 5, 4, 3, 6).reshape(-1, H, t * TILE, P, 2)
        out.append((c * sz[..., :1] + sz[..., 1:]).reshape(*lead, H, t * TILE, P * 64))
    return out


def _rotate(x, table, pos, kind=torch.float32):
    """Rotary embedding of x [T, heads, D] at pos, pairs (i, i + D/2), rounded to bf16 as the framework stores it."""
    cs = table[pos.long()].to(kind)[:, None]
    a, b = x.to(kind).chunk(2, -1)
    c, s = cs[..., 0], cs[..., 1]
    return torch.cat([a * c - b * s, b * c + a * s], -1).to(torch.bfloat16)


# ------------------------------------------------------------------------------------------------ the operators, plain
def _tables(state):
    case, page, T = state["case"], state["case"]["page"], state["T"]
    rows, want, lens, table, free = state["rows"].long(), state["want"].long(), state["lens"], state["block_table"], state["free_pages"]
    R, max_pages = rows.shape[0], table.shape[1]
    old = lens[rows].long()
    have, need = (old + page - 1) // page, (want + page - 1) // page
    # pages given back go on top of the stack, in batch order; then pages are taken from the top, in batch order
    back = (have - need).clamp(min=0)
    col = torch.arange(max_pages, device=DEV)
    entries = table[rows].long()
    n_free = state["n_free"].long()
    given = (col >= need[:, None]) & (col < have[:, None])
    at = n_free + (back.cumsum(0) - back)[:, None] + col - need[:, None]
    stack = torch.cat([free.long(), free.new_zeros(1, dtype=torch.long)])
    stack.scatter_(0, torch.where(given, at, free.shape[0]).flatten(), entries.flatten())
    stack = stack[:-1]
    top = n_free + back.sum()
    take = (need - have).clamp(min=0)
    upto = take.cumsum(0)
    fits = (take == 0) | (upto <= top)
    taken = (col >= have[:, None]) & (col < need[:, None]) & fits[:, None]
    entries = torch.where(taken, stack[(top - 1 - (upto - take)[:, None] - (col - have[:, None])).clamp(0, free.shape[0] - 1)], entries)
    block_table = table.index_copy(0, rows, entries.int())
    new = (want - old).clamp(min=0)
    cu = torch.cat([new.new_zeros(1), new.cumsum(0)])
    req = torch.repeat_interleave(torch.arange(R, device=DEV), new, output_size=T)
    pos = old[req] + torch.arange(T, device=DEV) - cu[req]
    slot = torch.where(fits[req], entries[req, pos // page] * page + pos % page, -1)
    kv_len = torch.where(fits, want, 0)
    return {"block_table": block_table, "free_pages": stack.int(), "lens": lens.index_copy(0, rows, torch.where(fits, want, old).int()),
            "n_free": (top - torch.where(fits, take, 0).sum()).int(), "refused": (~fits).sum().int().reshape(1), "cu_q": cu.int(),
            "kv_len": kv_len.int(), "slot": slot.int(), "pos": torch.where(fits[req], pos, -1).int()}


def _append(state):
    page, H = state["case"]["page"], state["case"]["H"]
    k = _rotate(state["k"], state["rope"], state["pos"])
    slot = state["slot"].long()
    # the bytes of every token's tile positions, written where the format has them
    pages, n = state["pages"], slot.shape[0]
    kc, ks, kz = _quantise(k.float())
    vc, vs, vz = _quantise(state["v"].float())
    P = kc.shape[2]
    p, tile, i = slot // page, slot % page // TILE, slot % TILE
    lane = torch.arange(512, device=DEV)
    g, t, j, c = lane[::2] // 64, lane[::2] // 16 % 4, lane[::2] // 4 % 4, lane[::2] // 2 % 2
    key = ((i % 8)[:, None] * 4 + torch.arange(4, device=DEV)) * 16                       # first bytes of the token's four lanes
    w = torch.arange(4, device=DEV) * 4
    kbyte = (key[:, :, None, None] + w[:, None] + 2 * torch.arange(2, device=DEV) + (i // 8)[:, None, None, None])     # token, t, j, c
    kval = kc.reshape(n, H, P, 4, 2, 4, 2).permute(0, 1, 2, 5, 3, 6, 4)                   # token, head, plane, t, j, c, half
    vlane = (torch.arange(8, device=DEV) * 4 + (i % 8 // 2)[:, None]) * 16                # token, g
    vbyte = 512 + vlane[:, :, None] + w + (2 * (i % 2) + i // 8)[:, None, None]           # token, g, j
    vval = vc.reshape(n, H, P, 4, 2, 8).permute(0, 1, 2, 5, 3, 4)                         # token, head, plane, g, j, half
    h, q = torch.arange(H, device=DEV)[:, None], torch.arange(P, device=DEV)
    put = lambda b: (p[:, None, None, None], h[..., None], tile[:, None, None, None], q[:, None], b[:, None, None])  # noqa: E731
    pages[put(kbyte.flatten(1))] = (kval[..., 0] | (kval[..., 1] << 4)).reshape(n, H, P, 32)
    pages[put(vbyte.flatten(1))] = (vval[..., 0] | (vval[..., 1] << 4)).reshape(n, H, P, 32)
    pair = torch.stack([torch.stack([ks, kz], -1), torch.stack([vs, vz], -1)], -2).to(torch.bfloat16).view(torch.uint8)   # token, head, plane, kv, 4
    pbyte = 1024 + (i % 8)[:, None, None] * 16 + torch.arange(2, device=DEV)[:, None] * 8 + (i // 8)[:, None, None] * 4 + torch.arange(4, device=DEV)
    pages[put(pbyte.flatten(1))] = pair.reshape(n, H, P, 8)
    # and back
    kk, vv = _unpack(pages[p, :, tile][:, :, None])
    at = i[:, None, None, None].expand(-1, H, 1, kk.shape[-1])
    return {"k": kk.gather(2, at)[:, :, 0].to(torch.bfloat16), "v": vv.gather(2, at)[:, :, 0].to(torch.bfloat16)}


def _attention(state, kind=torch.float32):
    case = state["case"]
    R, heads, H, D, page = case["R"], case["heads"], case["H"], case["D"], case["page"]
    G, nq, T = heads // H, state["max_q"], state["T"]
    cu, kv_len = state["cu_q"].long(), state["kv_len"].long()
    q_len = cu[1:] - cu[:-1]
    req = torch.repeat_interleave(torch.arange(R, device=DEV), q_len, output_size=T)
    at = torch.arange(T, device=DEV) - cu[req]
    pos = (kv_len - q_len)[req] + at
    q = torch.zeros(R, nq, heads, D, dtype=kind, device=DEV)
    q[req, at] = _rotate(state["q"], state["rope"], pos, kind).to(kind)
    q = q.reshape(R, nq, H, G, D).permute(0, 2, 1, 3, 4).reshape(R, H, nq * G, D)
    n = (state["max_kv"] + page - 1) // page
    b = state["pages"][state["block_table"][:, :n].long()]                       # R, n, H, tiles, planes, bytes
    k, v = _unpack(b.transpose(1, 2).reshape(R, H, n * (page // TILE), D // 64, TILE_BYTES), kind)
    s = torch.matmul(q, k.transpose(-1, -2)).mul_(1 / math.sqrt(D))
    last = (kv_len - q_len)[:, None] + torch.arange(nq, device=DEV)              # last key that a query sees
    seen = torch.arange(k.shape[2], device=DEV) <= last.repeat_interleave(G, 1)[..., None]
    s.masked_fill_(~seen[:, None], -math.inf)
    s.sub_(s.amax(-1, keepdim=True)).exp_()
    o = torch.matmul(s, v) / s.sum(-1, keepdim=True)
    return o.reshape(R, H, nq, G, D).permute(0, 2, 1, 3, 4).reshape(R, nq, heads, D)[req, at]


def run(state):
    kind = state["case"]["kind"]
    if own:
        import paper_2410_09687_b200 as moin
        if kind == "tables":
            b = moin.kv_update(state["tables"], state["want"], state["batch"], rows=state["rows"], lens_out=state["lens_out"],
                               n_free_out=state["n_free_out"])
            return {"block_table": state["block_table"], "free_pages": state["free_pages"], "lens": state["lens_out"],
                    "n_free": state["n_free_out"], "refused": b.refused, "cu_q": b.cu_q, "kv_len": b.kv_len, "slot": b.slot, "pos": b.pos}
        if kind == "append":
            moin.kv_append(state["cache"], state["slot"], state["k"], state["v"], pos=state["pos"], rope=state["rope"])
            k, v = moin.kv_read(state["cache"], state["slot"])
            return {"k": k, "v": v}
        return moin.kv_attention(state["cache"], state["tables"], state["q"], state["cu_q"], state["kv_len"], state["max_q"],
                                 state["max_kv"], rope=state["rope"])
    if kind == "tables":
        return _tables(state)
    if kind == "append":
        return _append(state)
    return _attention(state).to(torch.bfloat16)


def work(case):
    old, new = _lengths(case)
    R, page, T = case["R"], case["page"], int(new.sum())
    if case["kind"] == "tables":
        grown = int((_pages(old + new, page) - _pages(old, page)).sum())
        # rows, wanted and held lengths, pages off the stack; lengths, offsets, pages, and slot and position of every token
        return {"bytes": 4 * (3 * R + grown + 3 * R + grown + 2 * T), "flops": 0}
    row = case["H"] * case["D"] // 64 * 72        # bytes of a cached token: 64 codes and two pairs, keys and values
    if case["kind"] == "append":
        values = T * case["H"] * case["D"] * 4    # a key and a value of two bytes each
        return {"bytes": 2 * values + 2 * T * row + 8 * T + T * case["D"] * 4, "flops": T * case["H"] * case["D"] * 16}
    seen = int((new * (old + new) - new * (new - 1) // 2).sum())
    return {"bytes": int((old + new).sum()) * row + 4 * T * case["heads"] * case["D"] + T * case["D"] * 4
            + 4 * int(_pages(old + new, page).sum()), "flops": 4 * case["heads"] * case["D"] * seen}


# ------------------------------------------------------------------------------------------------ the same in 64 bits
def exact(case, seed):
    """Tables: a walk over the requests, one page at a time.  Append: rows quantised from the definition in numpy.  Attention:
    codes looked up byte by byte as the format describes them, softmax and sums in 64 bits, a request at a time."""
    state = prepare(case, seed)
    host = lambda n: state[n].cpu().numpy().astype(np.int64)  # noqa: E731
    page = case["page"]
    if case["kind"] == "tables":
        table, lens, stack = host("block_table"), host("lens"), host("free_pages")
        rows, want, n = host("rows"), host("want"), int(host("n_free")[0])
        for r, w in zip(rows, want):
            for p in range(-(-w // page), -(-lens[r] // page)):
                stack[n] = table[r, p]
                n += 1
        left, asked, refused, cu, kv, slot, pos = n, 0, 0, [0], [], [], []
        for r, w in zip(rows, want):
            have, need = -(-lens[r] // page), -(-w // page)
            asked += max(0, need - have)
            ok = need <= have or asked <= n
            for p in range(have, need if ok else have):
                left -= 1
                table[r, p] = stack[left]
            at = np.arange(lens[r], max(w, lens[r]))
            slot.append(table[r, at // page] * page + at % page if ok else np.full(at.size, -1))
            pos.append(at if ok else np.full(at.size, -1))
            cu.append(cu[-1] + at.size)
            kv.append(w if ok else 0)
            refused += not ok
            lens[r] = w if ok else lens[r]
        whole = lambda a: np.asarray(a, np.int32)  # noqa: E731
        return {"block_table": whole(table), "free_pages": whole(stack), "lens": whole(lens), "n_free": whole([left]), "refused": whole([refused]),
                "cu_q": whole(cu), "kv_len": whole(kv), "slot": whole(np.concatenate(slot)), "pos": whole(np.concatenate(pos))}
    bf16 = lambda a: torch.from_numpy(a).to(torch.bfloat16).double().numpy()  # noqa: E731

    def turn(x, pos):
        cs = state["rope"].double().cpu().numpy()[pos][:, None]
        half = x.shape[-1] // 2
        a, b = x[..., :half], x[..., half:]
        return bf16(np.concatenate([a * cs[..., 0] - b * cs[..., 1], b * cs[..., 0] + a * cs[..., 1]], -1))

    if case["kind"] == "append":
        out = {}
        for name in ("k", "v"):
            x = state[name].double().cpu().numpy()
            x = turn(x, host("pos")) if name == "k" else x
            x = x.reshape(*x.shape[:-1], -1, 64)
            lo = x.min(-1, keepdims=True)
            scale = bf16(np.maximum(np.maximum((x.max(-1, keepdims=True) - lo) / 15, np.abs(lo) / 4096), 2.0 ** -64))
            value = lo + scale * np.clip(np.rint((x - lo) / scale), 0, 15)
            out[name] = torch.from_numpy(value.reshape(*state[name].shape))
        return out
    # attention: index of every (token of a tile, channel) in the tile's bytes, and which half of the byte
    tok, ch = np.meshgrid(np.arange(16), np.arange(64), indexing="ij")
    j, half, low = ch // 16, ch // 8 % 2, ch % 8
    kbyte = (((tok % 8) * 4 + low // 2) * 4 + j) * 4 + 2 * (low % 2) + tok // 8
    vbyte = 512 + ((low * 4 + tok % 8 // 2) * 4 + j) * 4 + 2 * (tok % 2) + tok // 8
    pair = 1024 + (np.arange(16) % 8) * 16 + np.arange(16) // 8 * 4
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(DEV)  # noqa: E731
    byte, shift, pair = [dev(kbyte), dev(vbyte)], dev(4 * half), dev(pair)
    G, H, D = case["heads"] // case["H"], case["H"], case["D"]
    cu, kv_len, table = host("cu_q"), host("kv_len"), host("block_table")
    out = torch.zeros(state["T"], case["heads"], D, dtype=torch.float64)
    for r in range(case["R"]):
        n, nq = int(kv_len[r]), int(cu[r + 1] - cu[r])
        if nq == 0:
            continue
        b = state["pages"][dev(table[r, :-(-n // page)])]                        # pages, H, tiles, planes, bytes
        kv = []
        for which in range(2):
            code = (b[..., byte[which]].int() >> shift) & 15                     # pages, H, tiles, planes, 16, 64
            word = [b[..., pair + 8 * which + i].int() for i in range(4)]
            scale = ((word[0] | word[1] << 8) << 16).view(torch.float32).double()
            zero = ((word[2] | word[3] << 8) << 16).view(torch.float32).double()
            x = zero[..., None] + scale[..., None] * code
            kv.append(x.permute(1, 0, 2, 4, 3, 5).reshape(H, -1, D)[:, :n])
        pos = np.arange(n - nq, n)
        q = dev(turn(state["q"][cu[r]:cu[r + 1]].double().cpu().numpy(), pos)).reshape(nq, H, G, D).transpose(0, 1).reshape(H, nq * G, D)
        s = q @ kv[0].transpose(1, 2) / math.sqrt(D)
        s = torch.where(torch.arange(n, device=DEV) <= dev(pos).repeat_interleave(G)[:, None], s, -math.inf)
        o = torch.softmax(s, -1) @ kv[1]
        out[cu[r]:cu[r + 1]] = o.reshape(H, nq, G, D).transpose(0, 1).reshape(nq, case["heads"], D).cpu()
    return out
