"""The tree operators written out in numpy float64, one node at a time."""
import numpy as np

MIN_EXP = -100


def bf16_round(x):
    """Nearest bf16, ties to even (float64 in and out; normal range)."""
    m, e = np.frexp(np.asarray(x, np.float64))
    return np.ldexp(np.rint(np.ldexp(m, 8)), e - 8)


def e4m3_round(x):
    """Nearest e4m3 value of |x| <= 448, ties to even."""
    x = np.asarray(x, np.float64)
    _, e = np.frexp(x)
    step = np.ldexp(1.0, np.maximum(e - 1, -6) - 3)
    return np.rint(x / step) * step


def quantised(x):
    """(code values, exponents) of rows: the smallest e >= -100 with max |x| <= 448 2^e."""
    top = np.abs(x).max(-1)
    m, k = np.frexp(top)
    e = np.where(top > 0, k - 9 + (m > 0.875), MIN_EXP)
    e = np.maximum(e, MIN_EXP)
    return e4m3_round(np.ldexp(x, -e[..., None])), e


def rotated(x, pos, freq, layout, R, mscale):
    """x [..., D] at one position each."""
    x = np.asarray(x, np.float64)
    ang = np.asarray(pos, np.float64)[..., None] * freq
    c, s = np.cos(ang) * mscale, np.sin(ang) * mscale
    y = x.copy()
    for i in range(R // 2):
        a, b = (i, i + R // 2) if layout == "half" else (2 * i, 2 * i + 1)
        y[..., a] = x[..., a] * c[..., i] - x[..., b] * s[..., i]
        y[..., b] = x[..., b] * c[..., i] + x[..., a] * s[..., i]
    return y


def attention(q, clean, donor, gen, depth, visible, steps, LW, layer, window, scale, span):
    """(out, lse, spread, size) with q [C][T][Hq][D], clean / donor (k, v) [Hkv][Tp][D] (donor None: ZERO), gen (k, v)
    [C][Hkv][cap][D].  spread: sum p |v|, size: the largest scale * sum |q k| of a row's visible keys, n: their count.
    Rows that are not computed are NaN."""
    C, T, Hq, D = q.shape
    Hkv, Tp = clean[0].shape[:2]
    G, a, b = Hq // Hkv, span[0], span[1]
    out, spread = np.full(q.shape, np.nan), np.full(q.shape, np.nan)
    lse, size, n = (np.full((C, T, Hq), np.nan) for _ in range(3))
    for c in range(C):
        if steps[c] < 0:
            continue
        for t in range(T):
            if depth[c, t] < 0:
                continue
            d = min(int(depth[c, t]), T - 1)
            step = int(steps[c]) + d
            low = Tp + step - window + 1 if window else 0
            spliced = layer >= LW[c][0] and step >= LW[c][1]
            pos = [j for j in range(Tp) if j >= low]
            rows = [i for i in range(int(steps[c])) if Tp + i >= low]
            nodes = [u for u in range(T) if depth[c, u] >= 0 and (int(visible[c, t]) >> u) & 1 and
                     Tp + int(steps[c]) + min(int(depth[c, u]), T - 1) >= low]
            rows = rows + [int(steps[c]) + u for u in nodes]
            for h in range(Hq):
                g = h // G
                kv = []
                for x in range(2):
                    p = clean[x][g].copy()
                    if spliced:
                        p[a:b] = 0.0 if donor is None else donor[x][g, a:b]
                    kv.append(np.concatenate([p[pos], gen[x][c, g, rows]]).reshape(-1, D))
                K, V = kv
                n[c, t, h] = len(K)
                if len(K) == 0:
                    out[c, t, h], lse[c, t, h], spread[c, t, h], size[c, t, h] = 0.0, -np.inf, 0.0, 0.0
                    continue
                s = scale * (K @ q[c, t, h])
                m = s.max()
                p = np.exp(s - m)
                z = p.sum()
                lse[c, t, h] = m + np.log(z)
                out[c, t, h] = (p / z) @ V
                spread[c, t, h] = (p / z) @ np.abs(V)
                size[c, t, h] = scale * (np.abs(K) @ np.abs(q[c, t, h])).max()
    return out, lse, spread, size, n


def attention_bounds(out, lse, spread, size, n, D):
    """How far a kernel may be off: fp32 dot products of D terms (relative to the sum of magnitudes) move a score by
    D 2^-24 size and a weight by as much; exp2, the running sums of n weights and the division add (n + 16) 2^-24; P
    is rounded to bf16 (2^-8), and so is the result (2^-8)."""
    score = (D + 4) * 2.0 ** -24 * size
    rel = 2 * score + (n + 16) * 2.0 ** -24
    return ((2.0 ** -8 + 2 * rel[..., None]) * spread * (1 + 2.0 ** -8) + 2.0 ** -8 * np.abs(out) + 2.0 ** -126,
            score + (n + 16) * 2.0 ** -24 + 2.0 ** -22 * (1 + np.where(np.isfinite(lse), np.abs(lse), 0)))


def scores(x, tokens, k):
    """(logp, lse, entropy, rank, top, top_logp) of rows x (already scaled, float64), raw order given by x itself."""
    rows, vocab = x.shape
    got = [np.full(rows, np.nan), np.full(rows, np.nan), np.full(rows, np.nan), np.full(rows, -1), np.zeros((rows, k), int),
           np.full((rows, k), np.nan)]
    for r in range(rows):
        v = x[r]
        key = np.where(np.isnan(v), np.inf, v)
        order = sorted(range(vocab), key=lambda i: (not np.isnan(v[i]), -key[i], i))
        got[4][r] = order[:k]
        t = int(tokens[r])
        if 0 <= t < vocab:
            got[3][r] = order.index(t)
        if np.isnan(v).any():
            continue
        m = v.max()
        if m == -np.inf:
            got[1][r] = -np.inf
            continue
        if m == np.inf:
            continue
        e = np.exp(v - m)
        got[1][r] = m + np.log(e.sum())
        p = e / e.sum()
        with np.errstate(all="ignore"):
            got[2][r] = np.where(p > 0, p * (got[1][r] - v), 0).sum()
        if 0 <= t < vocab:
            got[0][r] = v[t] - got[1][r]
        got[5][r] = v[got[4][r]] - got[1][r]
    return got
