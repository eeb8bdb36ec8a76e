"""Performance cases of the operators that judge a tree of drafted tokens per sweep cell in one pass.

A case is one call of one operator of ``paper_2605_30574_amd`` over synthetic inputs of the shapes
in ``workloads/configs.py`` (attention) and ``workloads/model.py`` (vocabularies):

  attn     splice_tree_attn: the attention of every cell's T drafted tokens over its spliced
           prompt, its generated rows and the tree's own rows;
  append   splice_tree_append: rotary positions of T new tokens and their K/V written to the
           caches, bf16 or 8 bits (then read back by splice_tree_read);
  keep     splice_tree_keep: the cache rows of the accepted nodes moved together;
  scores   splice_token_scores: log probability, entropy, rank and top alternatives of given tokens.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DEV = "cuda"
SINK = 50.0            # sink outlier: prompt position 0, channels 0..3 of K
MIN_EXP, BIAS = -100, 127   # smallest exponent of an 8-bit row, bias of its byte

# attention shapes: (Hq, Hkv, D)
QWEN, GEMMA, TINY = (32, 8, 128), (8, 4, 256), (4, 2, 64)


def _attn(heads, **kw):
    c = dict(op="attn", Hq=heads[0], Hkv=heads[1], D=heads[2], layer=9, n_layers=36, window=0, donor="diff", kv="bf16",
             unit_scale=False)
    c.update(kw)
    return c


def _append(heads, **kw):
    c = dict(op="append", Hq=heads[0], Hkv=heads[1], D=heads[2], Tp=8192, layout="half", rotary=heads[2], theta=1e6,
             factor=1.0, mscale=1.0, kv="bf16", fused_qkv=True)
    c.update(kw)
    return c


def _keep(heads, **kw):
    c = dict(op="keep", Hkv=heads[1], D=heads[2], kv="bf16")
    c.update(kw)
    return c


def _scores(**kw):
    c = dict(op="scores", dtype="f32", k=8, pad=0, masked=0.0, scale=1.0, spread=2.0)
    c.update(kw)
    return c


def listed():
    return [
        # a chain of two tokens a cell over a short prompt with the ZERO donor: launch latency
        dict(_attn(TINY, C=6, T=2, Tp=32, a=4, b=28, cap=16, layer=1, n_layers=2, donor="zero"), name="attn_tiny_chain"),
        # one cell, a full tree, a long prompt: few rows, the keys are what is spread over the GPU
        dict(_attn(QWEN, C=1, T=64, Tp=8192, a=128, b=8128, cap=1024), name="attn_one_cell_tree"),
        # a sweep's cells with trees of 16: the shared prompt in matrix products
        dict(_attn(QWEN, C=48, T=16, Tp=8192, a=128, b=8128, cap=1024), name="attn_sweep_tree"),
        # short prompt, long generations in an 8-bit cache, small trees: the generated rows' bytes
        dict(_attn(QWEN, C=64, T=5, Tp=256, a=40, b=236, cap=4096, donor="blank", kv="e4m3"), name="attn_e4m3_long_rows"),
        # a local layer: sliding window, wide heads
        dict(_attn(GEMMA, C=40, T=12, Tp=4096, a=64, b=4064, cap=128, window=1024, layer=7, n_layers=34, donor="blank"),
             name="attn_window_wide_head"),
        # one token a cell appended to a bf16 cache, the fused projection's rows
        dict(_append(QWEN, C=32, T=1, cap=512), name="append_single"),
        # trees appended to an 8-bit cache, interleaved pairs on half of the head, frequencies scaled for a long context
        dict(_append(QWEN, C=128, T=33, cap=512, layout="interleaved", rotary=64, factor=8.0, mscale=1.1, kv="e4m3"),
             name="append_e4m3_partial"),
        # a few accepted tokens of small trees
        dict(_keep(QWEN, C=16, T=7, cap=256), name="keep_small"),
        # long accepted paths of a wide batch in an 8-bit cache
        dict(_keep(QWEN, C=128, T=64, cap=256, kv="e4m3"), name="keep_e4m3"),
        # a decode batch's last logits
        dict(_scores(rows=7, vocab=151936), name="scores_few_rows"),
        # every node of a sweep's trees, bf16 logits of a head product
        dict(_scores(rows=1024, vocab=128256, dtype="bf16", k=20), name="scores_trees_bf16"),
        # float32 logits with padded rows and masked vocabulary, probabilities at a temperature, no alternatives
        dict(_scores(rows=300, vocab=151936, pad=3, masked=0.2, scale=1.25, k=0), name="scores_masked_f32"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("attn", "attn", "attn", "append", "keep", "scores"))
    heads = rng.choice((QWEN, QWEN, GEMMA, TINY, (8, 8, 64), (16, 8, 128), (16, 2, 128)))
    kv = rng.choice(("bf16", "e4m3"))
    if op == "attn":
        C, T = _log(rng, 1, 96), _log(rng, 1, 64)
        Tp = 0 if rng.random() < 0.05 else _log(rng, 1, 8192)
        while C * T * heads[0] * (Tp + 512) > 48 * 16 * 32 * 8192:   # no more than the largest listed case
            C = (C + 1) // 2
            if C == 1:
                break
        a = rng.randint(0, Tp)
        return _attn(heads, C=C, T=T, Tp=Tp, a=a, b=rng.randint(a, Tp), cap=T + _log(rng, 1, 2048), kv=kv,
                     layer=rng.randint(0, 35), window=rng.choice((0, 0, _log(rng, 1, 2048))),
                     donor=rng.choice(("diff", "blank", "zero")), unit_scale=rng.random() < 0.2)
    if op == "append":
        T = _log(rng, 1, 64)
        return _append(heads, C=_log(rng, 1, 128), T=T, cap=T + _log(rng, 1, 512), Tp=_log(rng, 1, 131072), kv=kv,
                       layout=rng.choice(("half", "interleaved")), rotary=rng.choice((heads[2], heads[2] // 2, heads[2] // 4)),
                       theta=rng.choice((1e4, 5e5, 1e6)), factor=rng.choice((1.0, 4.0, 8.0)), mscale=rng.choice((1.0, 1.2)),
                       fused_qkv=rng.random() < 0.7)
    if op == "keep":
        T = _log(rng, 1, 64)
        return _keep(heads, C=_log(rng, 1, 128), T=T, cap=T + _log(rng, 1, 512), kv=kv)
    vocab = _log(rng, 3, 160000)
    rows = max(1, min(_log(rng, 1, 1024), 1024 * 128256 // vocab))
    return _scores(rows=rows, vocab=vocab, dtype=rng.choice(("f32", "bf16")), k=min(vocab, rng.choice((0, 1, 5, 20, 64))),
                   pad=rng.choice((0, 0, 1, 8)), masked=rng.choice((0.0, 0.3)), scale=rng.choice((1.0, 0.7, 1.4)),
                   spread=rng.choice((0.5, 2.0, 6.0)))


# ---------------------------------------------------------------- inputs

def _gen(seed, n):
    return torch.Generator(device=DEV).manual_seed((int(seed) * 7919 + n) % (1 << 62))


def _randn(seed, n, *shape, dtype=torch.bfloat16):
    return torch.randn(*shape, generator=_gen(seed, n), device=DEV, dtype=torch.float32).to(dtype)


def _tree(rng, C, T):
    """Random trees: node 0 is the root, a node's parent comes before it; some cells have fewer nodes (depth -1)."""
    depth, words = np.full((C, T), -1, np.int32), np.zeros((C, T), np.uint64)
    for c in range(C):
        n = T if c % 3 else int(rng.integers((T + 1) // 2, T + 1))
        for t in range(n):
            parent = -1 if t == 0 else int(rng.integers(max(0, t - 4), t))
            depth[c, t] = 0 if parent < 0 else depth[c, parent] + 1
            words[c, t] = (np.uint64(0) if parent < 0 else words[c, parent]) | np.uint64(1 << t)
    return torch.from_numpy(depth).to(DEV), torch.from_numpy(words.view(np.int64)).to(DEV)


def _steps(rng, C, T, cap):
    s = rng.integers(0, cap - T + 1, size=C).astype(np.int32)
    s[0] = cap - T
    if C >= 8:
        s[C // 2] = -1   # a finished cell
    return s


def _cells(rng, C, n_layers, steps):
    """Cutoffs and onsets of a sweep: some cells never spliced, some from their first step, some in the middle of the tree."""
    L = rng.integers(0, n_layers + 1, size=C)
    W = rng.integers(0, 64, size=C)
    W[1::4] = 0
    W[2::4] = np.maximum(steps[2::4], 0) + 1
    return np.ascontiguousarray(np.stack([L, W], 1).astype(np.int32))


def _empty_cache(case, seed, n):
    """A generated cache [C][Hkv][cap][D] with rows in it: (codes or bf16, exponent bytes or None)."""
    shape = (case["C"], case["Hkv"], case["cap"], case["D"])
    x = torch.randn(*shape, generator=_gen(seed, n), device=DEV, dtype=torch.float32)
    if case["kv"] == "bf16":
        return x.to(torch.bfloat16), None
    e = torch.randint(BIAS - 10, BIAS - 5, shape[:3], generator=_gen(seed, n + 50), device=DEV).to(torch.uint8)
    return (x * 90).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8), e


def prepare(case, seed):
    rng = np.random.default_rng(int(seed) % (1 << 62))
    s = dict(case=case)
    op = case["op"]
    if op == "scores":
        rows, vocab = case["rows"], case["vocab"]
        x = torch.randn(rows, vocab + case["pad"], generator=_gen(seed, 1), device=DEV, dtype=torch.float32) * case["spread"]
        x.scatter_add_(1, torch.randint(0, vocab, (rows, 4), generator=_gen(seed, 2), device=DEV),
                       torch.full((rows, 4), 4.0, device=DEV))   # a few likely tokens
        if case["masked"]:
            x[:, int(vocab * (1 - case["masked"])):] = -math.inf
        dtype = torch.float32 if case["dtype"] == "f32" else torch.bfloat16
        s["logits"] = x.to(dtype)[:, :vocab]
        s["tokens"] = torch.randint(0, max(1, int(vocab * (1 - case["masked"]))), (rows,), generator=_gen(seed, 3), device=DEV)
        s["out"] = [torch.empty(rows, device=DEV) for _ in range(3)] + [torch.empty(rows, dtype=torch.int64, device=DEV)]
        if case["k"]:
            s["out"] += [torch.empty(rows, case["k"], dtype=torch.int64, device=DEV), torch.empty(rows, case["k"], device=DEV)]
        if own:
            import paper_2605_30574_amd as sp
            s["workspace"] = torch.empty(sp.splice_token_scores_workspace_bytes(rows, vocab, case["k"]), dtype=torch.uint8, device=DEV)
        return s
    C, T, Hkv, D = case["C"], case["T"], case["Hkv"], case["D"]
    steps = _steps(rng, C, T, case["cap"])
    s["steps"] = steps
    s["steps_dev"] = torch.from_numpy(steps).to(DEV)
    s["depth"], s["visible"] = _tree(rng, C, T)
    s["k"], s["ke"] = _empty_cache(case, seed, 10)
    s["v"], s["ve"] = _empty_cache(case, seed, 11)
    if own:
        import paper_2605_30574_amd as sp
        s["shape"] = sp.make_shape(C, case.get("n_layers", 1), case.get("Hq", Hkv), Hkv, D, case.get("Tp", 0),
                                   (case.get("a", 0), case.get("b", 0)), case["cap"], case.get("donor") == "zero", "bf16")
        s["tree"] = sp.make_tree(T, case["kv"])
    if op == "keep":
        # accepted nodes: the root's path, ascending
        keep = np.full((C, T), -1, np.int32)
        for c in range(C):
            n = int(rng.integers(0, T + 1))
            keep[c, :n] = np.sort(rng.choice(T, size=n, replace=False))
        s["keep"] = torch.from_numpy(keep).to(DEV)
        return s
    Hq = case["Hq"]
    if op == "append":
        if case["fused_qkv"]:   # one projection's rows, q, k and v side by side
            qkv = _randn(seed, 1, C, T, (Hq + 2 * Hkv) * D)
            s["q"], s["kn"], s["vn"] = (x.unflatten(2, (-1, D)) for x in
                                        qkv.split((Hq * D, Hkv * D, Hkv * D), dim=2))
        else:
            s["q"], s["kn"], s["vn"] = (_randn(seed, 1 + i, C, T, h, D) for i, h in enumerate((Hq, Hkv, Hkv)))
        R = case["rotary"]
        s["freq"] = (case["theta"] ** (-torch.arange(0, R, 2, dtype=torch.float64) / R) / case["factor"]).to(DEV)
        s["q_out"] = torch.zeros(C, T, Hq, D, dtype=torch.bfloat16, device=DEV)
        s["rows_k"] = torch.zeros(C, Hkv, T, D, dtype=torch.bfloat16, device=DEV)
        s["rows_v"] = torch.zeros_like(s["rows_k"])
        if own:
            s["rope"] = sp.make_rope(case["layout"], R, case["mscale"])
        return s
    Tp, a, b = case["Tp"], case["a"], case["b"]
    s["q"] = _randn(seed, 1, C, T, Hq, D)
    fold = 1 / math.sqrt(D) if case["unit_scale"] else 1.0

    def prompt(n):
        k, v = _randn(seed, n, Hkv, Tp, D, dtype=torch.float32) * fold, _randn(seed, n + 1, Hkv, Tp, D)
        k[:, :1, :4] *= SINK
        return k.to(torch.bfloat16), v

    s["ck"], s["cv"] = prompt(20)
    s["dk"] = s["dv"] = None
    if case["donor"] != "zero":
        s["dk"], s["dv"] = prompt(22)
        if case["donor"] == "blank":   # only the span is another
            for x, y in (("dk", "ck"), ("dv", "cv")):
                s[x][:, :a], s[x][:, b:] = s[y][:, :a], s[y][:, b:]
    s["LW"] = _cells(rng, C, case["n_layers"], steps)
    s["scale"] = 1.0 if case["unit_scale"] else 1 / math.sqrt(D)
    s["out"] = torch.zeros(C, T, Hq, D, dtype=torch.bfloat16, device=DEV)
    s["lse"] = torch.zeros(C, T, Hq, device=DEV)
    if own:
        s["call"] = sp.make_call(case["layer"], 0, case["window"], s["scale"])
        s["workspace"] = torch.empty(sp.splice_tree_attn_workspace_bytes(s["shape"], s["call"], s["tree"]), dtype=torch.uint8,
                                     device=DEV)
    return s


# ---------------------------------------------------------------- plain forms

def _values(codes, e):
    """float32 values of a cache: bf16, or 8-bit codes with a power of two a row."""
    if e is None:
        return codes.float()
    return codes.view(torch.float8_e4m3fn).float() * torch.exp2(e.float() - BIAS)[..., None]


def _quantised(x):
    """(codes, exponent bytes) of float32 rows."""
    m, k = torch.frexp(x.abs().amax(-1))
    e = torch.clamp(k - 9 + (m > 0.875).to(torch.int32), min=MIN_EXP)
    return torch.ldexp(x, -e[..., None]).to(torch.float8_e4m3fn).view(torch.uint8), (e + BIAS).to(torch.uint8)


def _plain_attn(s):
    c = s["case"]
    C, T, Hq, Hkv, D, Tp, a, b = (c[x] for x in ("C", "T", "Hq", "Hkv", "D", "Tp", "a", "b"))
    G, steps, depth = Hq // Hkv, s["steps_dev"][:, None], s["depth"]
    valid = (depth >= 0) & (steps >= 0)                                        # [C, T]
    step = steps + depth
    LW = torch.from_numpy(s["LW"]).to(DEV)
    spliced = (LW[:, :1] <= c["layer"]) & (step >= LW[:, 1:])
    low = Tp + step - c["window"] + 1 if c["window"] else torch.zeros_like(step)   # the first position a query sees
    q = s["q"].float().view(C, T, Hkv, G, D)
    # the prompt, shared by the cells
    qp = q.permute(2, 0, 1, 3, 4).reshape(Hkv, C * T * G, D)
    sp = torch.matmul(qp, s["ck"].float().transpose(1, 2).contiguous()).view(Hkv, C, T, G, Tp)
    pick = spliced[None, :, :, None, None]
    if s["dk"] is None:
        sp[..., a:b] = torch.where(pick, 0.0, sp[..., a:b])
    else:
        sd = torch.matmul(qp, s["dk"][:, a:b].float().transpose(1, 2).contiguous()).view(Hkv, C, T, G, b - a)
        sp[..., a:b] = torch.where(pick, sd, sp[..., a:b])
        del sd
    sp.mul_(s["scale"])
    seen = torch.arange(Tp, device=DEV) >= low[..., None]                       # [C, T, Tp]
    sp.masked_fill_(~seen[None, :, :, None, :], -math.inf)
    # the cell's own rows and the tree's
    n = min(c["cap"], int(s["steps"].max()) + T)
    gk, gv = (_values(s[x][:, :, :n], None if s[e] is None else s[e][:, :, :n]) for x, e in (("k", "ke"), ("v", "ve")))
    qg = q.permute(0, 2, 1, 3, 4).reshape(C, Hkv, T * G, D)
    sg = torch.matmul(qg, gk.transpose(2, 3).contiguous()).view(C, Hkv, T, G, n).mul_(s["scale"])
    row = torch.arange(n, device=DEV)
    j = torch.clamp(row - steps, 0, T - 1)                                      # [C, n]: the tree's node of a row
    committed = (row < steps)[:, None] & (Tp + row >= low[..., None])
    node_depth = torch.gather(depth, 1, j)[:, None]
    drafted = ((row >= steps) & (row < steps + T))[:, None] & (node_depth >= 0) & (Tp + steps[..., None] + node_depth >= low[..., None])
    drafted = drafted & ((s["visible"][..., None] >> j[:, None]) & 1).bool()
    sg.masked_fill_(~(committed | drafted)[:, None, :, None, :], -math.inf)
    # one softmax over both
    sg_p = sg.permute(1, 0, 2, 3, 4)
    m = sg_p.amax(-1)
    if Tp:
        m = torch.maximum(m, sp.amax(-1))
    m = torch.where(m == -math.inf, 0.0, m)                                     # [Hkv, C, T, G]
    sp = sp.sub_(m[..., None]).exp_()
    sg = sg.sub_(m.permute(1, 0, 2, 3)[..., None]).exp_()
    l = sp.sum(-1) + sg.sum(-1).permute(1, 0, 2, 3)
    o = torch.matmul(sg.view(C, Hkv, T * G, n), gv).view(C, Hkv, T, G, D).permute(1, 0, 2, 3, 4)
    if s["dk"] is None:
        sp[..., a:b] = torch.where(pick, 0.0, sp[..., a:b])
    else:
        dv = s["dv"][:, a:b].float()
        o = o + torch.matmul(torch.where(pick, sp[..., a:b], 0.0).view(Hkv, C * T * G, b - a), dv).view(Hkv, C, T, G, D)
        sp[..., a:b] = torch.where(pick, 0.0, sp[..., a:b])
    o = o + torch.matmul(sp.view(Hkv, C * T * G, Tp), s["cv"].float()).view(Hkv, C, T, G, D)
    o = torch.where(l[..., None] > 0, o / l[..., None], 0.0)
    lse = m + torch.log(l)
    out = o.permute(1, 2, 0, 3, 4).reshape(C, T, Hq, D).to(torch.bfloat16)
    lse = lse.permute(1, 2, 0, 3).reshape(C, T, Hq)
    return {"out": torch.where(valid[..., None, None], out, s["out"]), "lse": torch.where(valid[..., None], lse, s["lse"])}


def _rotated(x, cos, sin, case):
    """Rotary positions of x [C][T][H][D] (float32); cos, sin [C][T][R / 2]."""
    R = case["rotary"]
    cos, sin, part = cos[:, :, None], sin[:, :, None], x[..., :R]
    if case["layout"] == "half":
        u, v = part[..., :R // 2], part[..., R // 2:]
        turned = torch.cat([u * cos - v * sin, v * cos + u * sin], -1)
    else:
        u, v = part[..., 0::2], part[..., 1::2]
        turned = torch.stack([u * cos - v * sin, v * cos + u * sin], -1).flatten(-2)
    return torch.cat([turned, x[..., R:]], -1)


def _plain_append(s):
    c = s["case"]
    C, T, Hkv, D = c["C"], c["T"], c["Hkv"], c["D"]
    steps, depth = s["steps_dev"][:, None], s["depth"]
    valid = ((depth >= 0) & (steps >= 0))[..., None, None]                      # [C, T, 1, 1]
    ang = (c["Tp"] + steps + depth).double()[..., None] * s["freq"]
    cos, sin = (f(ang).float() * c["mscale"] for f in (torch.cos, torch.sin))
    q = _rotated(s["q"].float(), cos, sin, c).to(torch.bfloat16)
    k, v = _rotated(s["kn"].float(), cos, sin, c), s["vn"].float()
    s["q_out"].copy_(torch.where(valid, q, s["q_out"]))
    at = torch.clamp(steps, min=0) + torch.arange(T, device=DEV)                # [C, T]: a node's row
    cell = torch.arange(C, device=DEV)[:, None]
    got = {"q": s["q_out"]}
    for x, name, e in ((k, "k", "ke"), (v, "v", "ve")):
        cache = s[name]
        if s[e] is None:
            cache[cell, :, at] = torch.where(valid, x.to(torch.bfloat16), cache[cell, :, at])
            got[name] = cache
            continue
        codes, ex = _quantised(x)
        cache[cell, :, at] = torch.where(valid, codes, cache[cell, :, at])
        s[e][cell, :, at] = torch.where(valid[..., 0], ex, s[e][cell, :, at])
        got[name] = cache.view(torch.float8_e4m3fn)
        rows = _values(cache[cell, :, at], s[e][cell, :, at]).to(torch.bfloat16).transpose(1, 2)
        s["rows_" + name].copy_(torch.where((steps >= 0)[..., None, None], rows, s["rows_" + name]))
        got["rows_" + name] = s["rows_" + name]
    return got


def _plain_keep(s):
    c = s["case"]
    C, T = c["C"], c["T"]
    steps = s["steps_dev"][:, None]
    base, node = torch.clamp(steps, min=0), torch.arange(T, device=DEV)
    frm = base + torch.where((s["keep"] >= 0) & (steps >= 0), s["keep"], node)
    cell, got = torch.arange(C, device=DEV)[:, None], {}
    for name, e in (("k", "ke"), ("v", "ve")):
        s[name][cell, :, base + node] = s[name][cell, :, frm]
        got[name] = s[name]
        if s[e] is not None:
            s[e][cell, :, base + node] = s[e][cell, :, frm]
            got[name], got[e] = s[name].view(torch.float8_e4m3fn), s[e]
    return got


def _plain_scores(s):
    c = s["case"]
    logits, tokens = s["logits"].float(), s["tokens"]
    x = logits * c["scale"]
    m = x.amax(-1, keepdim=True)
    z = x - m
    e = torch.exp(z)
    l = e.sum(-1)
    log_l = torch.log(l)
    entropy = log_l - (e * torch.where(e > 0, z, 0.0)).sum(-1) / l
    lse = m[:, 0] + log_l
    xt = torch.gather(x, 1, tokens[:, None])
    raw = torch.gather(logits, 1, tokens[:, None])
    ids = torch.arange(c["vocab"], device=DEV)
    rank = ((logits > raw) | ((logits == raw) & (ids < tokens[:, None]))).sum(-1)
    got = {"logp": xt[:, 0] - lse, "lse": lse, "entropy": entropy, "rank": rank}
    if c["k"]:
        bits = (logits + 0.0).view(torch.int32)   # in the order of the values, the lower index first among equals
        key = torch.where(bits < 0, bits ^ 0x7fffffff, bits).long() * (1 << 24) + ((1 << 24) - 1 - ids)
        top = (1 << 24) - 1 - (torch.topk(key, c["k"], dim=-1).values & ((1 << 24) - 1))
        got["top"], got["top_logp"] = top, torch.gather(x, 1, top) - lse[:, None]
    return got


def _own(s):
    import paper_2605_30574_amd as sp
    c = s["case"]
    if c["op"] == "scores":
        o = s["out"]
        top = o[4:] if c["k"] else (None, None)
        sp.splice_token_scores(s["logits"], s["tokens"], o[0], o[1], o[2], o[3], top[0], top[1], s["workspace"], scale=c["scale"])
        got = {"logp": o[0], "lse": o[1], "entropy": o[2], "rank": o[3]}
        if c["k"]:
            got["top"], got["top_logp"] = top
        return got
    if c["op"] == "attn":
        sp.splice_tree_attn(s["shape"], s["call"], s["tree"], s["LW"], s["steps"], s["depth"], s["visible"], s["q"], s["ck"],
                            s["cv"], s["dk"], s["dv"], s["k"], s["v"], s["ke"], s["ve"], s["out"], s["lse"], s["workspace"])
        return {"out": s["out"], "lse": s["lse"]}
    if c["op"] == "keep":
        sp.splice_tree_keep(s["shape"], s["tree"], s["steps"], s["keep"], s["k"], s["v"], s["ke"], s["ve"])
        if s["ke"] is None:
            return {"k": s["k"], "v": s["v"]}
        return {"k": s["k"].view(torch.float8_e4m3fn), "ke": s["ke"], "v": s["v"].view(torch.float8_e4m3fn), "ve": s["ve"]}
    sp.splice_tree_append(s["shape"], s["tree"], s["rope"], s["freq"], s["steps"], s["depth"], s["q"], s["kn"], s["vn"],
                          s["q_out"], s["k"], s["v"], s["ke"], s["ve"])
    if s["ke"] is None:
        return {"q": s["q_out"], "k": s["k"], "v": s["v"]}
    sp.splice_tree_read(s["shape"], s["tree"], s["steps"], s["k"], s["v"], s["ke"], s["ve"], s["rows_k"], s["rows_v"])
    return {"q": s["q_out"], "k": s["k"].view(torch.float8_e4m3fn), "rows_k": s["rows_k"], "v": s["v"].view(torch.float8_e4m3fn),
            "rows_v": s["rows_v"]}


def run(state):
    if own:
        return _own(state)
    return {"attn": _plain_attn, "append": _plain_append, "keep": _plain_keep, "scores": _plain_scores}[state["case"]["op"]](state)


# ---------------------------------------------------------------- what a pass cannot do without

def work(case):
    op = case["op"]
    if op == "scores":
        n = case["rows"] * case["vocab"]
        return {"bytes": n * (4 if case["dtype"] == "f32" else 2) + case["rows"] * (8 + 20 + 12 * case["k"]), "flops": 4 * n}
    C, T, Hkv, D, cap = (case[x] for x in ("C", "T", "Hkv", "D", "cap"))
    active = C - 1 if C >= 8 else C
    row = D * 2 if case["kv"] == "bf16" else D + 1                              # bytes of a cached row
    if op == "keep":
        return {"bytes": 2 * 2 * active * (T / 2) * Hkv * row, "flops": 0}
    Hq = case["Hq"]
    if op == "append":
        n = active * T
        back = 0 if case["kv"] == "bf16" else 2 * n * Hkv * (row + 2 * D)
        return {"bytes": n * (2 * D * (2 * Hq + 2 * Hkv) + 2 * Hkv * row) + back, "flops": 3 * n * (Hq + Hkv) * case["rotary"]}
    w = case["window"]
    seen_p = case["Tp"] if not w else max(0, min(case["Tp"], w - cap // 2))
    seen_g = (cap - T) / 2 if not w else min(w, (cap - T) / 2)
    span = 0 if case["donor"] == "zero" else min(seen_p, case["b"] - case["a"])
    return {"bytes": 2 * Hkv * D * 2 * (seen_p + span) + 2 * active * Hkv * (seen_g + T) * row + active * T * Hq * (4 * D + 4),
            "flops": 4 * active * T * Hq * D * (seen_p + seen_g + T / 2)}


# ---------------------------------------------------------------- the definitions in 64 bits

def _e4m3(x):
    """x (float64) to the nearest 8-bit value, ties to even: 3 bits behind the leading one, steps of 2^-9 below 2^-6."""
    step = torch.exp2(torch.clamp(torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -40))), min=-6) - 3)
    return torch.round(x / step) * step


def _exact_attn(s):
    c = s["case"]
    C, T, Hq, Hkv, D, Tp, a, b, w = (c[x] for x in ("C", "T", "Hq", "Hkv", "D", "Tp", "a", "b", "window"))
    G = Hq // Hkv
    depth, words = s["depth"].cpu().numpy(), s["visible"].cpu().numpy().view(np.uint64)
    out, lse = s["out"].double(), s["lse"].double()
    clean = [s[x].double() for x in ("ck", "cv")]
    donor = [torch.zeros_like(x) if c["donor"] == "zero" else s[y].double() for x, y in zip(clean, ("dk", "dv"))]
    spliced = [torch.cat([x[:, :a], y[:, a:b], x[:, b:]], 1) for x, y in zip(clean, donor)]
    for n in range(C):
        s0 = int(s["steps"][n])
        if s0 < 0:
            continue
        rows = []
        for x, e in (("k", "ke"), ("v", "ve")):
            r = s[x][n, :, :s0 + T]
            rows.append(r.double() if s[e] is None else
                        r.view(torch.float8_e4m3fn).double() * 2.0 ** (s[e][n, :, :s0 + T].double() - BIAS)[..., None])
        for kind in (False, True):
            nodes = [t for t in range(T) if depth[n, t] >= 0 and
                     (c["layer"] >= s["LW"][n, 0] and s0 + depth[n, t] >= s["LW"][n, 1]) == kind]
            if not nodes:
                continue
            K, V = (torch.cat([p, r], 1) for p, r in zip(spliced if kind else clean, rows))
            at = torch.tensor(nodes, device=DEV)
            q = s["q"][n, at].double().view(len(nodes), Hkv, G, D).permute(1, 0, 2, 3).reshape(Hkv, -1, D)
            x = torch.bmm(q, K.transpose(1, 2).contiguous()).view(Hkv, len(nodes), G, -1) * s["scale"]
            see = np.zeros((len(nodes), Tp + s0 + T), bool)
            for i, t in enumerate(nodes):
                p = Tp + s0 + depth[n, t]
                see[i, :Tp + s0] = np.arange(Tp + s0) > (p - w if w else -1)
                for u in range(T):
                    see[i, Tp + s0 + u] = depth[n, u] >= 0 and (int(words[n, t]) >> u) & 1 and (not w or depth[n, t] - depth[n, u] < w)
            x = x.masked_fill(~torch.from_numpy(see).to(DEV)[None, :, None], -math.inf)
            z = torch.logsumexp(x, -1)
            p = torch.exp(x - torch.where(z == -math.inf, 0.0, z)[..., None])
            o = torch.bmm(p.view(Hkv, -1, p.shape[-1]), V).view(Hkv, len(nodes), G, D)
            out[n, at] = o.permute(1, 0, 2, 3).reshape(len(nodes), Hq, D)
            lse[n, at] = z.permute(1, 0, 2).reshape(len(nodes), Hq)
    return {"out": out, "lse": lse}


def _exact_append(s):
    c = s["case"]
    R, T = c["rotary"], c["T"]
    depth, steps = s["depth"].cpu().numpy(), s["steps"]
    i = torch.arange(c["D"], device=DEV)
    if c["layout"] == "half":
        other, sign = torch.where(i < R // 2, i + R // 2, i - R // 2), torch.where(i < R // 2, -1.0, 1.0).double()
        pair = torch.where(i < R // 2, i, i - R // 2)
    else:
        other, sign, pair = i ^ 1, torch.where(i % 2 == 0, -1.0, 1.0).double(), i // 2
    other, pair = torch.where(i < R, other, i), torch.where(i < R, pair, 0)
    got = {"q": s["q_out"].double()}
    for name, e in (("k", "ke"), ("v", "ve")):
        got[name] = s[name].double() if s[e] is None else s[name].view(torch.float8_e4m3fn).double()
        if s[e] is not None:
            got["rows_" + name] = s["rows_" + name].double()
    for n in range(c["C"]):
        s0 = int(steps[n])
        if s0 < 0:
            continue
        if s["ke"] is not None:   # rows that padding leaves are read back as they were
            for name, e in (("k", "ke"), ("v", "ve")):
                old = s[name][n, :, s0:s0 + T].view(torch.float8_e4m3fn).double()
                got["rows_" + name][n] = old * 2.0 ** (s[e][n, :, s0:s0 + T].double() - BIAS)[..., None]
        at = torch.tensor([t for t in range(T) if depth[n, t] >= 0], dtype=torch.long, device=DEV)
        ang = (c["Tp"] + s0 + s["depth"][n, at]).double()[:, None] * s["freq"][pair]
        cos, sin = torch.cos(ang) * c["mscale"], torch.sin(ang) * c["mscale"] * sign
        cos, sin = torch.where(i < R, cos, 1.0)[:, None], torch.where(i < R, sin, 0.0)[:, None]
        turn = lambda x: x * cos + x[..., other] * sin  # noqa: E731
        got["q"][n, at] = turn(s["q"][n, at].double())
        for name, e, x in (("k", "ke", turn(s["kn"][n, at].double())), ("v", "ve", s["vn"][n, at].double())):
            if s[e] is None:
                got[name][n, :, s0 + at] = x.transpose(0, 1)
                continue
            top = x.abs().amax(-1, keepdim=True)
            ex = torch.clamp(torch.ceil(torch.log2(top / 448)), min=MIN_EXP)
            code = _e4m3(x / torch.exp2(ex))
            got[name][n, :, s0 + at] = code.transpose(0, 1)
            got["rows_" + name][n, :, at] = (code * torch.exp2(ex)).transpose(0, 1)
    return got


def _exact_keep(s):
    c = s["case"]
    keep, got = s["keep"].cpu().numpy(), {}
    for name, e in (("k", "ke"), ("v", "ve")):
        got[name] = s[name].clone() if s[e] is None else s[name].view(torch.float8_e4m3fn).float()
        got[name] = got[name].double()
        if s[e] is not None:
            got[e] = None
        for n in range(c["C"]):
            s0, path = int(s["steps"][n]), [int(t) for t in keep[n] if t >= 0]
            if s0 >= 0 and path:
                at = torch.tensor(path, device=DEV)
                got[name][n, :, s0:s0 + len(path)] = got[name][n, :, s0 + at]
    return got


def _exact_scores(s):
    c = s["case"]
    got = {"logp": [], "lse": [], "entropy": [], "rank": None}
    if c["k"]:
        got["top"], got["top_logp"] = None, []
    for r in range(c["rows"]):
        raw = s["logits"][r].double()
        x = raw * c["scale"]
        z = torch.logsumexp(x, 0)
        p = torch.exp(x - z)
        got["lse"].append(z)
        got["logp"].append(x[s["tokens"][r]] - z)
        got["entropy"].append(torch.where(p > 0, p * (z - x), 0.0).sum())
        if c["k"]:
            got["top_logp"].append(torch.sort(x, descending=True).values[:c["k"]] - z)
    return {k: torch.stack(v) if isinstance(v, list) else v for k, v in got.items()}


def exact(case, seed):
    s = prepare(case, seed)
    return {"attn": _exact_attn, "append": _exact_append, "keep": _exact_keep, "scores": _exact_scores}[case["op"]](s)
