"""The definitions behind the paged entries (splice_pages.h) in plain numpy float64, byte by byte and cell by cell."""
import math

import numpy as np

LEVELS = np.array([0, .5, 1, 1.5, 2, 3, 4, 6])
VALUES = np.concatenate([LEVELS, -LEVELS])
P = 64


def head_bytes(D):
    return 68 * D


def places(r, d, D):
    """Where token r keeps value d of a head: (K byte, V byte, K scale, V scale); the value's half of the byte is d % 2."""
    n = min(4, D // 32)
    a, e, c, f = r // 32, r // 16 % 2, r // 4 % 4, r % 4
    b, i, g = d // 64, d % 64 // 4, d % 4 // 2
    block = d // 32
    v = (((((a * (D // 64) + b) * 4 + c) * 16 + i) * 2 + e) * 4 + f) * 2 + g
    ks = ((block // n * 16 + r % 16) * n + block % n) * 4 + r // 16
    vs = ((((a * 4 + c) * 2 + block % 2) * (D // 64) + block // 2) * 2 + e) * 4 + f
    return r * (D // 2) + d // 2, 32 * D + v, 64 * D + ks, 66 * D + vs


def quantised(x):
    """(codes, exponents) of rows x [..., D]: codes [..., D] 0..15, exponents [..., D / 32] (None where not finite)."""
    blocks = x.reshape(*x.shape[:-1], -1, 32)
    top = np.abs(blocks).max(-1)
    e = np.maximum(np.floor(np.log2(np.maximum(top, 2.0 ** -120))).astype(int) - 4, -100)   # from below
    while (more := top > 6 * 2.0 ** e).any():
        e[more] += 1
    y = blocks / 2.0 ** e[..., None]
    order = np.abs(np.abs(y)[..., None] - LEVELS)              # distance to every level; of two nearest the even code
    least = order.min(-1, keepdims=True)
    code = np.where(order == least, np.arange(8) % 2 * 8 + np.arange(8), 99).argmin(-1)
    code = np.where((e >= 126)[..., None], np.minimum(code, 5), code)
    return (code + 8 * np.signbit(y)).reshape(x.shape), e


def dequantised(codes, e):
    return VALUES[codes] * np.repeat(2.0 ** e.astype(np.float64), 32, -1)


def page_of(k, v):
    """Bytes [68 D] of 64 rows' k, v [64][D] (finite)."""
    D = k.shape[-1]
    out = np.zeros(head_bytes(D), np.uint8)
    r, d = np.arange(P)[:, None], np.arange(D)
    (kc, ke), (vc, ve) = quantised(k), quantised(v)
    kb, vb, ks, vs = (np.broadcast_to(x, (P, D)) for x in places(r, d, D))
    for codes, at in ((kc, kb), (vc, vb)):
        out[at[:, 0::2]] = codes[:, 0::2] + 16 * codes[:, 1::2]
    for e, at in ((ke, ks), (ve, vs)):
        out[at[:, 0::32]] = e + 127
    return out


def rows_of(page, D):
    """(k, v) float64 [64][D] of a page's bytes; NaN where the exponent byte is 255."""
    r, d = np.arange(P)[:, None], np.arange(D)
    kb, vb, ks, vs = (np.broadcast_to(x, (P, D)) for x in places(r, d, D))
    got = []
    for codes, scale in ((kb, ks), (vb, vs)):
        byte = page[codes].astype(int)
        code = np.where(d % 2 == 1, byte >> 4, byte & 15)
        e = page[scale].astype(np.float64)
        got.append(np.where(e == 255, np.nan, VALUES[code] * 2.0 ** (np.minimum(e, 254) - 127)))
    return got


def attend(q, keys, values, scale):
    """(out [D], lse, sum of weights |value| [D], the largest scale sum |q||k|) of one query over keys [n][D]."""
    if len(keys) == 0:
        return np.zeros(q.shape), -math.inf, np.zeros(q.shape), 0.0
    x = keys @ q * scale
    m = x.max()
    w = np.exp(x - m)
    z = w.sum()
    return (w / z) @ values, m + math.log(z), (w / z) @ np.abs(values), (np.abs(keys) @ np.abs(q)).max() * scale


def fork(parent, rows, want, tables, refs, n_pages):
    """(tables, refs, missing, copied) after splice_page_fork."""
    C, L = tables.shape
    held, need = -(-rows // P), -(-want // P)
    new, refs = np.full((C, L), -1), refs.astype(np.int64).copy()
    ok = lambda p: 0 <= p < n_pages  # noqa: E731
    for c in range(C):
        for j in range(L):
            if ok(tables[c, j]):
                refs[tables[c, j]] -= 1
            if parent[c] >= 0 and j < held[c] and ok(tables[parent[c], j]):
                new[c, j] = tables[parent[c], j]
                refs[new[c, j]] += 1
    last = [new[c, held[c] - 1] if rows[c] % P else -1 for c in range(C)]
    copies = [last[c] >= 0 and not (refs[last[c]] == last.count(last[c]) and last.index(last[c]) == c) for c in range(C)]
    for c in range(C):
        if copies[c]:
            refs[last[c]] -= 1
    free = [p for p in range(n_pages) if refs[p] == 0]
    missing, copied = 0, np.full((C, 2), -1)
    for c in range(C):
        for j in ([held[c] - 1] if copies[c] else []) + list(range(held[c], need[c])):
            new[c, j] = free.pop(0) if free else -1
            if new[c, j] < 0:
                missing += 1
                continue
            refs[new[c, j]] = 1
            if copies[c] and j == held[c] - 1:
                copied[c] = last[c], new[c, j]
    return new, refs, missing, copied


def kept(keep, limit):
    """The entries of a keep list [T] up to where it ends."""
    got = []
    for k in keep:
        if k < 0 or (got and k <= got[-1]) or k >= limit:
            break
        got.append(int(k))
    return got
