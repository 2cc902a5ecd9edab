"""Keys and values in 4 bits: the format, its pages, the page plan and the
attention over the pages, in fp64 (plain loops over requests, heads and rows).
"""
import numpy as np

LEVELS = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def kv4_quantise(x):
    """(codes uint8 [..., d], scales uint8 [..., d / 32]) of fp64 [..., d]: per
    32 channels the least e in [-125, 125] with no magnitude above 7 * 2^e, the
    nearest level (ties to the even code); 255 where a value is not finite."""
    x = np.asarray(x, dtype=np.float64)
    g = x.reshape(*x.shape[:-1], x.shape[-1] // 32, 32)
    finite = np.isfinite(g).all(-1)
    y = np.where(finite[..., None], g, 0.0)
    most = np.abs(y).max(-1)
    e = np.full(most.shape, -125)
    while True:
        grow = (most > 7 * np.exp2(e.astype(np.float64))) & (e < 125)
        if not grow.any():
            break
        e = e + grow
    a = np.abs(y) / np.exp2(e.astype(np.float64))[..., None]
    dist = np.abs(a[..., None] - LEVELS)
    best = dist.min(-1, keepdims=True)
    order = np.array([0, 2, 4, 6, 1, 3, 5, 7])  # even codes first among the nearest
    code = order[np.argmax((dist == best)[..., order], -1)]
    code = code + 8 * np.signbit(y)
    scale = np.where(finite, e + 127, 255)
    return code.reshape(x.shape).astype(np.uint8), scale.astype(np.uint8)


def kv4_values(code, scale):
    """fp64 values of codes [..., d] and scales [..., d / 32]."""
    v = LEVELS[code & 7] * np.where(code & 8, -1.0, 1.0)
    s = np.where(scale == 255, np.nan, np.exp2(scale.astype(np.float64) - 127))
    return (v.reshape(*code.shape[:-1], code.shape[-1] // 32, 32) * s[..., None]).reshape(code.shape)


def _at(block, d, which, t, c):
    """Byte of channel c of token t in a head's part of a page; which: "kc",
    "ks", "vc", "vs"."""
    codes, scales = block * d // 2, block * d // 32
    if which == "kc":
        return t * (d // 2) + c // 2
    if which == "ks":
        return codes + t * (d // 32) + c // 32
    if which == "vc":
        return codes + scales + ((t // 8) * (d // 2) + c // 2) * 8 + t % 8
    return 2 * codes + scales + ((t // 8) * (d // 32) + c // 32) * 8 + t % 8


def kv4_store(pool, k, v, slots, block):
    """Writes the rows of k and v (fp64 [rows, heads, d]) into a pool uint8
    [pages, heads, bytes], in place."""
    _, heads, d = k.shape
    limit = pool.shape[0] * block
    c = np.arange(d)
    for row, slot in enumerate(slots):
        if not 0 <= slot < limit:
            continue
        page, t = divmod(int(slot), block)
        for h in range(heads):
            for x, which in ((k, "k"), (v, "v")):
                code, scale = kv4_quantise(x[row, h])
                pool[page, h, _at(block, d, which + "c", t, c[::2])] = code[::2] | (code[1::2] << 4)
                pool[page, h, _at(block, d, which + "s", t, c[::32])] = scale
    return pool


def kv4_token(pool, page, h, t, block, d):
    """(k, v) fp64 [d] of token t of a page."""
    c = np.arange(d)
    out = []
    for which in ("k", "v"):
        b = pool[page, h, _at(block, d, which + "c", t, c)]
        code = np.where(c % 2, b >> 4, b & 15).astype(np.uint8)
        out.append(kv4_values(code, pool[page, h, _at(block, d, which + "s", t, c[::32])]))
    return out


def kv4_cached(pool, table_row, kv_len, block, d):
    """(k, v fp64 [heads, tokens, d], there bool [tokens]) of one request."""
    n_pages, heads, _ = pool.shape
    n = min(max(int(kv_len), 0), len(table_row) * block)
    k, v = np.zeros((2, heads, n, d))
    there = np.zeros(n, dtype=bool)
    for t in range(n):
        page = int(table_row[t // block])
        if 0 <= page < n_pages:
            there[t] = True
            for h in range(heads):
                k[h, t], v[h, t] = kv4_token(pool, page, h, t % block, block, d)
    return k, v, there


def kv4_attention(q, pool, table, q_start, kv_len, block, causal=False, scale=0.0):
    """(o fp64 [rows, heads, d], lse [rows, heads], done bool [rows]); rows of
    no request are not done."""
    rows, heads, d = q.shape
    group = heads // pool.shape[1]
    sigma = scale if scale > 0 else 1.0 / np.sqrt(d)
    o, lse = np.zeros((rows, heads, d)), np.full((rows, heads), -np.inf)
    done = np.zeros(rows, dtype=bool)
    start = np.clip(np.asarray(q_start), 0, rows)
    for b in range(len(kv_len)):
        m = start[b + 1] - start[b]
        if m <= 0:
            continue
        k, v, there = kv4_cached(pool, table[b], kv_len[b], block, d)
        n = k.shape[1]
        done[start[b]:start[b] + m] = True
        for i in range(m):
            seen = there & ((np.arange(n) <= n - m + i) if causal else True)
            if not seen.any():
                continue
            for h in range(heads):
                with np.errstate(invalid="ignore"):
                    s = sigma * (k[h // group, seen] @ q[start[b] + i, h])
                    top = s.max()
                    p = np.exp(s - top)
                    o[start[b] + i, h] = p @ v[h // group, seen] / p.sum()
                    lse[start[b] + i, h] = top + np.log(p.sum())
    return o, lse, done


def page_plan(kv_len, new_len, table, free_pages, block, n_slots):
    """(q_start, kv_len_out, slots, positions, counts, table) by walking the
    new tokens one by one."""
    table = np.array(table, copy=True)
    batch, width = table.shape
    q_start, kv_out = [0], []
    slots, positions = np.full(n_slots, -1, np.int64), np.full(n_slots, -1, np.int64)
    taken = lacking = wanted = 0
    for b in range(batch):
        kv = min(max(int(kv_len[b]), 0), width * block)
        n = max(int(new_len[b]), 0)
        fits = min(n, n_slots - q_start[-1])
        placed = 0
        for i in range(fits):
            pos = kv + i
            at = q_start[-1] + i
            positions[at] = pos
            j = pos // block
            if j >= width:
                continue
            if pos % block == 0:
                wanted += 1
                if wanted <= len(free_pages):
                    table[b, j] = free_pages[wanted - 1]
                    taken += 1
            # a page entered before the call, or one the list had
            if j < -(-kv // block) or wanted <= len(free_pages):
                placed += 1
                if table[b, j] >= 0:
                    slots[at] = int(table[b, j]) * block + pos % block
        q_start.append(q_start[-1] + fits)
        kv_out.append(kv + placed)
        lacking += n - placed
    return np.array(q_start), np.array(kv_out), slots, positions, np.array([q_start[-1], taken, min(lacking, 2 ** 31 - 1)]), table
