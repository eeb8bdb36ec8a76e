"""The tree entries on the CPU: exports, refusals on the host before any device work, tree layouts, frequencies.
(No compute call runs here: there is no GPU.)"""
import ctypes
import math
import os
import re

import numpy as np
import pytest

import paper_2605_30574_amd as sp
from paper_2605_30574_amd import tree as T

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FAKE = 0x10000   # never dereferenced: every call here is refused, or has nothing to do


def test_library_exports_every_declared_symbol():
    text = open(os.path.join(ROOT, "include", "splice_tree.h")).read()
    declared = set(re.findall(r"SPLICE_API\s+[\w\s\*]+?\b(splice_\w+)\s*\(", text))
    assert declared == set(T.EXPORTS)
    lib = sp.load_library()
    for name in declared:
        assert hasattr(lib, name) and hasattr(sp, name), name


def shape(**kw):
    base = dict(n_cells=3, n_layers=4, n_q_heads=8, n_kv_heads=2, head_dim=64, prompt_len=32, span=(4, 28), gen_capacity=16,
                donor_zero=False, dtype="bf16")
    base.update(kw)
    return sp.make_shape(**base)


def ints(*x):
    return (ctypes.c_int32 * len(x))(*x)


STEPS, LW = ints(0, 5, -1), ints(0, 0, 1, 2, 9, 0)


def attn(sh=None, call=None, tree=None, LW=LW, steps=STEPS, **kw):
    a = dict(depth=FAKE, visible=FAKE, q=FAKE, ck=FAKE, cv=FAKE, dk=FAKE, dv=FAKE, gk=FAKE, gv=FAKE, gke=None, gve=None, out=FAKE,
             lse=FAKE, ws=FAKE, bytes=1 << 40)
    a.update(kw)
    sh, call, tree = sh or shape(), call or sp.make_call(1, 0, 0, 0.125), tree or sp.make_tree(4)
    return T._library().splice_tree_attn(ctypes.byref(sh), ctypes.byref(call), ctypes.byref(tree), LW, steps, *a.values(), None)


def append(sh=None, tree=None, rope=None, steps=STEPS, **kw):
    a = dict(depth=FAKE, pos=None, freq=FAKE, q=FAKE, qs=512, k=FAKE, ks=128, v=FAKE, vs=128, q_out=2 * FAKE, gk=FAKE, gv=FAKE,
             gke=None, gve=None)
    a.update(kw)
    sh, tree, rope = sh or shape(), tree or sp.make_tree(4), rope or sp.make_rope("half", 64)
    return T._library().splice_tree_append(ctypes.byref(sh), ctypes.byref(tree), ctypes.byref(rope), steps, *a.values(), None)


def keep(sh=None, tree=None, steps=STEPS, **kw):
    a = dict(keep=FAKE, gk=FAKE, gv=FAKE, gke=None, gve=None)
    a.update(kw)
    return T._library().splice_tree_keep(ctypes.byref(sh or shape()), ctypes.byref(tree or sp.make_tree(4)), steps, *a.values(), None)


def read(sh=None, tree=None, steps=STEPS, **kw):
    a = dict(gk=FAKE, gv=FAKE, gke=None, gve=None, rk=FAKE, rv=FAKE)
    a.update(kw)
    return T._library().splice_tree_read(ctypes.byref(sh or shape()), ctypes.byref(tree or sp.make_tree(4)), steps, *a.values(), None)


def scores(rows=3, vocab=100, k=5, stride=100, scale=1.0, dtype=sp.SPLICE_F32, **kw):
    a = dict(logits=FAKE, tokens=FAKE, logp=FAKE, lse=FAKE, entropy=FAKE, rank=FAKE, top=FAKE, top_logp=FAKE, ws=FAKE, bytes=1 << 40)
    a.update(kw)
    return T._library().splice_token_scores(a["logits"], dtype, rows, vocab, stride, scale, a["tokens"], k, a["logp"], a["lse"],
                                            a["entropy"], a["rank"], a["top"], a["top_logp"], a["ws"], a["bytes"], None)


EVERY = [attn, append, keep, read]


@pytest.mark.parametrize("entry", EVERY)
def test_shapes_trees_and_steps(entry):
    E4M3 = dict(gke=FAKE, gve=FAKE)
    assert entry(sh=shape(dtype="f32")) == sp.SPLICE_EUNSUPPORTED
    assert entry(sh=shape(head_dim=96)) == sp.SPLICE_EUNSUPPORTED
    assert entry(sh=shape(n_q_heads=6)) == sp.SPLICE_EUNSUPPORTED
    assert entry(sh=shape(span=(4, 33))) == sp.SPLICE_ESHAPE
    assert entry(tree=sp.make_tree(0)) == sp.SPLICE_ESHAPE
    assert entry(tree=sp.make_tree(65)) == sp.SPLICE_EUNSUPPORTED
    assert entry(tree=sp.make_tree(17)) == sp.SPLICE_ESHAPE               # more nodes than rows
    assert entry(tree=sp.SpliceTree(4, 2)) == sp.SPLICE_EINVAL
    assert entry(steps=None) == sp.SPLICE_EINVAL
    assert entry(steps=ints(0, 13, -1)) == sp.SPLICE_ESHAPE               # 13 + 4 > 16
    assert entry(steps=ints(0, 2**31 - 1, -1)) == sp.SPLICE_ESHAPE
    assert entry(gk=None) == sp.SPLICE_EINVAL
    assert entry(gv=None) == sp.SPLICE_EINVAL
    assert entry(gk=FAKE + 8) == sp.SPLICE_EINVAL
    assert entry(**E4M3) == sp.SPLICE_EINVAL                              # exponents with bf16 caches
    assert entry(tree=sp.make_tree(4, "e4m3")) == sp.SPLICE_EINVAL        # and none with 8-bit ones
    assert entry(tree=sp.make_tree(4, "e4m3"), gke=FAKE) == sp.SPLICE_EINVAL
    # nothing to do
    assert entry(steps=ints(-1, -7, -1)) == sp.SPLICE_OK
    assert entry(sh=shape(n_cells=0), steps=None) == sp.SPLICE_OK


@pytest.mark.parametrize("entry", EVERY)
def test_more_heads_than_a_grid_has_work_groups(entry):
    assert entry(sh=shape(n_q_heads=1 << 16, n_kv_heads=1 << 16)) == sp.SPLICE_EUNSUPPORTED
    assert entry(sh=shape(n_q_heads=1 << 30, n_kv_heads=1 << 30)) == sp.SPLICE_EUNSUPPORTED


def test_attention_refusals():
    assert attn(call=sp.make_call(1, 0, 0, 3e38)) == sp.SPLICE_EINVAL     # no float in base 2
    assert attn(call=sp.make_call(4, 0, 0, 0.1)) == sp.SPLICE_ESHAPE
    assert attn(call=sp.make_call(1, 0, -1, 0.1)) == sp.SPLICE_ESHAPE
    for scale in (0.0, -1.0, float("nan"), float("inf")):
        assert attn(call=sp.make_call(1, 0, 0, scale)) == sp.SPLICE_EINVAL
    assert attn(call=sp.make_call(1, 0, 0, 0.1, 65)) == sp.SPLICE_EINVAL
    assert attn(LW=None) == sp.SPLICE_EINVAL
    assert attn(LW=ints(0, 0, -1, 2, 9, 0)) == sp.SPLICE_ESHAPE
    for name in ("depth", "visible", "q", "ck", "cv", "dk", "dv", "out", "lse"):
        assert attn(**{name: None}) == sp.SPLICE_EINVAL, name
    for name in ("q", "ck", "cv", "dk", "dv", "gv", "out"):
        assert attn(**{name: FAKE + 8}) == sp.SPLICE_EINVAL, name
    for name, off in (("depth", 2), ("visible", 4), ("lse", 2)):
        assert attn(**{name: FAKE + off}) == sp.SPLICE_EINVAL, name
    assert attn(sh=shape(donor_zero=True)) == sp.SPLICE_EINVAL            # ZERO takes no buffers
    small = sp.make_call(1, 0, 0, 0.1, 64)
    sh = shape(prompt_len=4096)
    need = sp.splice_tree_attn_workspace_bytes(sh, small, sp.make_tree(4))
    assert need > 0
    assert attn(sh=sh, call=small, ws=None) == sp.SPLICE_EWORKSPACE
    assert attn(sh=sh, call=small, ws=FAKE + 16) == sp.SPLICE_EWORKSPACE
    assert attn(sh=sh, call=small, bytes=1024) == sp.SPLICE_EWORKSPACE


def test_workspace_refusals():
    assert T._library().splice_tree_attn_workspace_bytes(None, None, None) == sp.SPLICE_EINVAL
    sh, tree = shape(), sp.make_tree(4)
    assert T._library().splice_tree_attn_workspace_bytes(ctypes.byref(sh), None, ctypes.byref(tree)) == sp.SPLICE_EINVAL


def test_append_refusals():
    assert append(rope=sp.SpliceRope(2, 64, 1.0)) == sp.SPLICE_EINVAL
    assert append(rope=sp.make_rope("half", 64, float("nan"))) == sp.SPLICE_EINVAL
    for R in (-16, 8, 72, 80, 128):
        assert append(rope=sp.make_rope("half", R)) == sp.SPLICE_ESHAPE
    for name in ("depth", "q", "k", "v", "q_out", "freq"):
        assert append(**{name: None}) == sp.SPLICE_EINVAL, name
    for name, off in (("q", 8), ("k", 8), ("v", 8), ("q_out", 8), ("depth", 2), ("pos", 4), ("freq", 4)):
        assert append(**{name: FAKE + off}) == sp.SPLICE_EINVAL, name
    for name in ("qs", "ks", "vs"):
        for bad in (0, -512, 120, 516, 1 << 33):
            assert append(**{name: bad}) == sp.SPLICE_ESHAPE, (name, bad)
    assert append(q_out=FAKE, qs=768) == sp.SPLICE_EINVAL                 # in place over rows that are not dense


def test_keep_and_read_refusals():
    assert keep(keep=None) == sp.SPLICE_EINVAL
    assert keep(keep=FAKE + 2) == sp.SPLICE_EINVAL
    for name in ("rk", "rv"):
        assert read(**{name: None}) == sp.SPLICE_EINVAL
        assert read(**{name: FAKE + 8}) == sp.SPLICE_EINVAL


def test_scores_refusals():
    assert scores(dtype=2) == sp.SPLICE_EINVAL
    for kw in (dict(rows=-1), dict(vocab=0), dict(k=-1), dict(k=65), dict(vocab=4), dict(vocab=(1 << 28) + 1, stride=1 << 29),
               dict(rows=1 << 24), dict(stride=99), dict(stride=-100), dict(stride=1 << 33)):
        assert scores(**kw) == sp.SPLICE_ESHAPE, kw
    for scale in (0.0, -1.0, float("nan"), float("inf"), 3e38):
        assert scores(scale=scale) == sp.SPLICE_EINVAL
    for name in ("logits", "tokens", "logp", "lse", "entropy", "rank", "top", "top_logp"):
        assert scores(**{name: None}) == sp.SPLICE_EINVAL, name
        assert scores(**{name: FAKE + 1}) == sp.SPLICE_EINVAL, name
    assert scores(dtype=sp.SPLICE_BF16, logits=FAKE + 1) == sp.SPLICE_EINVAL
    need = sp.splice_token_scores_workspace_bytes(3, 100000, 5)
    assert need > 0
    for kw in (dict(ws=None), dict(bytes=need - 1), dict(ws=FAKE + 8)):
        assert scores(vocab=100000, stride=100000, **kw) == sp.SPLICE_EWORKSPACE
    assert scores(rows=0) == sp.SPLICE_OK
    with pytest.raises(sp.SpliceError):
        sp.splice_token_scores_workspace_bytes(1, 10, 11)


def test_binding_refuses_cpu_tensors():
    import torch
    sh, tree, call = shape(), sp.make_tree(4), sp.make_call(1, 0, 0, 0.1)
    x = torch.zeros(4)
    with pytest.raises(ValueError):
        sp.token_scores(torch.zeros(2, 9), torch.zeros(2, dtype=torch.int64))
    with pytest.raises(ValueError):
        sp.splice_tree_attn(sh, call, tree, [[0, 0]] * 3, [0, 0, 0], x, x, x, x, x, x, x, x, x, None, None, x, x, None)
    with pytest.raises(ValueError):
        sp.splice_tree_append(sh, tree, sp.make_rope("half", 64), x, [0, 0, 0], x, x, x, x, x, x, x)
    with pytest.raises(ValueError):
        sp.splice_tree_keep(sh, tree, [0, 0, 0], x, x, x)
    with pytest.raises(ValueError):
        sp.splice_tree_read(sh, tree, [0, 0, 0], x, x, None, None, x, x)


# ---------------------------------------------------------------- layouts and frequencies

def test_tree_layout():
    depth, words = sp.tree_layout([[-1, 0, 0, 1, 2, 3], [-1, -1, 1, -2, -2, -2]])
    assert depth.tolist() == [[0, 1, 1, 2, 2, 3], [0, 0, 1, -1, -1, -1]]
    assert words.tolist() == [[1, 3, 5, 11, 21, 43], [1, 2, 6, 0, 0, 0]]
    depth, words = sp.tree_layout(np.arange(-1, 63)[None])
    assert depth[0].tolist() == list(range(64)) and words[0, 63] == np.uint64(2**64 - 1)
    for bad in ([[0]], [[-1, 1]], [[-1, 2, 0]], [[-2, 0]], [[]], [list(range(-1, 64))], [-1, 0], [[-1.0]]):
        with pytest.raises(ValueError):
            sp.tree_layout(bad)


def test_frequencies():
    f, m = sp.rope_frequencies(64, 1e4)
    assert m == 1.0 and f.dtype == np.float64 and np.array_equal(f, 1e4 ** (-np.arange(0, 64, 2) / 64))
    g, m = sp.rope_frequencies(64, 1e4, "linear", 4.0)
    assert np.array_equal(g, f / 4) and m == 1.0
    # banded: fast pairs as they were, slow ones divided, between them between
    g, _ = sp.rope_frequencies(128, 5e5, "banded", 8.0, 8192)
    f, _ = sp.rope_frequencies(128, 5e5)
    wave = 2 * math.pi / f
    assert np.array_equal(g[wave < 8192 / 4], f[wave < 8192 / 4]) and np.allclose(g[wave > 8192], f[wave > 8192] / 8, rtol=1e-15)
    mid = (wave >= 8192 / 4) & (wave <= 8192)
    assert mid.any() and ((g[mid] <= f[mid]) & (g[mid] >= f[mid] / 8)).all()
    s = (8192 / wave[mid] - 1) / 3
    assert np.allclose(g[mid], (1 - s) * f[mid] / 8 + s * f[mid], rtol=1e-14)
    # yarn: over 32 turns within the original length as they were, under one divided
    g, m = sp.rope_frequencies(128, 1e6, "yarn", 4.0, 32768)
    f, _ = sp.rope_frequencies(128, 1e6)
    turns = 32768 * f / (2 * math.pi)
    assert m == pytest.approx(0.1 * math.log(4.0) + 1)
    first = np.flatnonzero(turns < 32)[0]
    assert np.array_equal(g[:first], f[:first])
    last = np.flatnonzero(turns < 1)[0]
    assert np.allclose(g[last + 1:], f[last + 1:] / 4, rtol=1e-14) and (np.diff(g) < 0).all()
    for kw in (dict(scaling="linear", factor=0.5), dict(scaling="other"), dict(scaling="yarn", factor=2.0), dict(scaling="banded"),
               dict(scaling="banded", original_len=100, low_freq_factor=4.0, high_freq_factor=1.0),
               dict(scaling="yarn", original_len=100, beta_fast=1.0, beta_slow=2.0)):
        with pytest.raises(ValueError):
            sp.rope_frequencies(64, 1e4, **kw)
    with pytest.raises(ValueError):
        sp.rope_frequencies(63, 1e4)
    assert sp.rope_frequencies(0, 1e4)[0].size == 0


def test_accepted_paths():
    from paper_2605_30574_amd.decode import accept
    parents = [[-1, -1, 0, 1, 1, 4], [-1, 0, 1, -2, -2, -2], [-1, 0, 0, 2, 3, 4]]
    tokens = [[7, 8, 9, 3, 4, 5], [1, 2, 3, 9, 9, 9], [6, 6, 6, 6, 6, 6]]
    best = [[9, 4, 0, 0, 5, 0], [2, 0, 0, 0, 0, 0], [6, 6, 6, 6, 6, 6]]
    keep, n = accept(parents, tokens, [8, 1, 5], best)
    assert keep.dtype == np.int32 and keep.tolist() == [[1, 4, 5, -1, -1, -1], [0, 1, -1, -1, -1, -1], [-1] * 6]
    assert n.tolist() == [3, 2, 0]
    assert accept(parents, tokens, [8, 1, 6], best)[0][2].tolist() == [0, 1, -1, -1, -1, -1]   # the lower of two children
