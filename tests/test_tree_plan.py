"""The host-side plan of splice_tree_attn (csrc/tree_plan.hpp), compiled here for the CPU: every item of the grid and every
partial result is where the kernels look for it, and the workspace that is asked for holds them."""
import ctypes
import os
import random
import subprocess

import pytest

import paper_2605_30574_amd as sp
from paper_2605_30574_amd import tree as T

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SRC = r"""
#include "tree_plan.hpp"
using namespace splice;
extern "C" {
int limits(int *r) { r[0] = kTreeMaxSlots; r[1] = kTreeMaxChunks; r[2] = kTreeMaxPrompt; return (int)sizeof(TreeSlots); }
// info [257], order [640], step [256], plan: n, row_waves, row_tiles, per, n_p, p_tiles, n_slots, blocks, most_chunks, split,
// p_heavy0, p_heavy
int64_t prepare(const splice_shape *sh, const splice_call *call, const splice_tree *tree, const int32_t *lw, const int32_t *steps,
                int n_cu, uint32_t *info, uint32_t *order, int32_t *step, int64_t *plan, int64_t *most) {
    if (validate_tree(sh, tree, steps) != SPLICE_OK) return -1;
    TreeSlots s{};
    int n = 0;
    const TreePlan p = tree_prepare(*sh, *call, *tree, lw, steps, n_cu, n, step, s);
    for (int i = 0; i <= SPLICE_MAX_CELLS; ++i) info[i] = s.info[i];
    for (int i = 0; i < kTreeMaxSlots; ++i) order[i] = (s.order[i / 2] >> (16 * (i % 2))) & 0xffff;
    const int64_t v[] = {n, p.row_waves, p.row_tiles, p.per, p.n_p, p.p_tiles, p.n_slots, p.blocks, p.most_chunks, p.split, p.p_heavy0, p.p_heavy};
    for (int i = 0; i < 12; ++i) plan[i] = v[i];
    *most = (int64_t)tree_most_bytes(*sh, *call, tree->n_nodes, n_cu);
    return (int64_t)p.bytes;
}
}
"""


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    d = tmp_path_factory.mktemp("tree_plan")
    src, so = d / "plan.cpp", d / "plan.so"
    src.write_text(SRC)
    subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-Wall", "-Werror", "-D_GLIBCXX_ASSERTIONS", "-fsanitize=undefined",
                    "-fno-sanitize-recover", "-I", os.path.join(ROOT, "include"), "-I", os.path.join(ROOT, "paper_2605_30574_amd", "csrc"),
                    "-o", str(so), str(src)], check=True)
    lib = ctypes.CDLL(str(so))
    lib.prepare.restype = ctypes.c_int64
    return lib


def draw(rng):
    log = lambda lo, hi: int(round(lo * (hi / lo) ** rng.random()))  # noqa: E731
    C, n = log(1, 256), log(1, 64)
    Hkv, G, D = rng.choice((1, 2, 4, 8, 32)), rng.choice((1, 2, 4, 8)), rng.choice((64, 128, 256))
    Tp = rng.choice((0, log(1, 100000)))
    cap = n + log(1, 100000)
    a = rng.randint(0, Tp)
    sh = sp.make_shape(C, 8, Hkv * G, Hkv, D, Tp, (a, rng.randint(a, Tp)), cap, rng.random() < 0.3, "bf16")
    call = sp.make_call(3, 0, rng.choice((0, 0, log(1, 5000))), 0.1, rng.choice((0, 0, 0, 64, 256, 65536)))
    steps = [rng.choice((-1, 0, cap - n, rng.randint(0, cap - n))) if rng.random() < 0.5 else rng.randint(0, cap - n) for _ in range(C)]
    lw = [(rng.randint(0, 8), rng.choice((0, max(s, 0) + rng.randint(0, 70), 10**9))) for s in steps]
    return sh, call, sp.make_tree(n, rng.choice(("bf16", "e4m3"))), lw, steps


def test_plans(plan):
    lim = (ctypes.c_int * 3)()
    assert plan.limits(lim) < 2600   # the kernels' arguments stay under 4 KiB
    slots_max, chunks_max, prompt_max = lim
    rng = random.Random(7)
    packed = split = 0
    for trial in range(3000):
        sh, call, tree, lw, steps = draw(rng)
        C, n_nodes = sh.n_cells, tree.n_nodes
        info, order, step = (ctypes.c_uint32 * 257)(), (ctypes.c_uint32 * slots_max)(), (ctypes.c_int32 * 256)()
        v, most = (ctypes.c_int64 * 12)(), ctypes.c_int64()
        flat = (ctypes.c_int32 * (2 * C))(*[x for p in lw for x in p])
        n_bytes = plan.prepare(ctypes.byref(sh), ctypes.byref(call), ctypes.byref(tree), flat, (ctypes.c_int32 * C)(*steps),
                               rng.choice((256, 304, 64)), info, order, step, v, ctypes.byref(most))
        n, row_waves, row_tiles, per, n_p, p_tiles, n_slots, blocks, most_chunks, is_split, heavy0, heavy = v
        active = [c for c in range(C) if steps[c] >= 0]
        assert n == len(active)
        if n == 0:
            continue
        packed, split = packed + (n_p > 0), split + is_split
        G = sh.n_q_heads // sh.n_kv_heads
        rows = n_nodes * G
        assert row_tiles * row_waves * 32 >= rows and row_waves in (1, 2, 4) and per >= 1
        assert sorted(info[i] & 255 for i in range(n)) == active
        onset = [(info[i] >> 8) & 255 for i in range(n)]
        first = [info[i] >> 16 for i in range(n + 1)]
        for i in range(n):
            c = info[i] & 255
            assert step[i] == steps[c]
            for d in range(n_nodes):   # the splice predicate, node by node
                assert (d >= onset[i]) == (call.layer >= lw[c][0] and steps[c] + d >= lw[c][1])
            assert 1 <= first[i + 1] - first[i] - n_p <= chunks_max and first[i + 1] - first[i] <= min(64, most_chunks)
        assert first[0] == 0 and first[n] == n_slots
        items = n_slots - n * n_p
        assert items <= slots_max and n_p <= prompt_max and blocks == row_tiles * items + n_p * p_tiles <= 65535
        assert not n_p or (p_tiles * 128 >= n * rows > (p_tiles - 1) * 128 and rows <= 64)
        if n_p:   # row tiles with unspliced and spliced nodes are among the heavy ones, which begin first
            assert 0 <= heavy0 and 0 <= heavy and heavy0 + heavy <= p_tiles
            for t in range(p_tiles):
                cells = range(t * 128 // rows, min((t * 128 + 127) // rows + 1, n))
                if any(onset[i] > 0 for i in cells) and any(onset[i] < 64 for i in cells):
                    assert heavy0 <= t < heavy0 + heavy
        seen = {(order[i] & 255, order[i] >> 8) for i in range(items)}
        assert seen == {(i, k) for i in range(n) for k in range(first[i + 1] - first[i] - n_p)}
        assert is_split == (n_slots > n)
        assert n_bytes == (n_slots * n_nodes * sh.n_q_heads * (2 * sh.head_dim + 16) if is_split else 0)
        assert n_bytes <= most.value
    assert packed > 300 and split > 1000


def test_python_asks_the_library_for_the_bytes():
    sh, call = sp.make_shape(8, 4, 8, 2, 64, 4096, (4, 28), 512, False, "bf16"), sp.make_call(1, 0, 0, 0.1)
    assert sp.splice_tree_attn_workspace_bytes(sh, call, sp.make_tree(4)) > 0
    with pytest.raises(sp.SpliceError):
        sp.splice_tree_attn_workspace_bytes(sh, call, T.SpliceTree(4, 9))


def plan_of(plan, sh, call, tree, lw, steps, n_cu=256):
    """The plan's values by name, and the workspace's bytes."""
    info, order, step = (ctypes.c_uint32 * 257)(), (ctypes.c_uint32 * 640)(), (ctypes.c_int32 * 256)()
    v, most = (ctypes.c_int64 * 12)(), ctypes.c_int64()
    flat = (ctypes.c_int32 * (2 * len(steps)))(*[x for p in lw for x in p])
    n_bytes = plan.prepare(ctypes.byref(sh), ctypes.byref(call), ctypes.byref(tree), flat, (ctypes.c_int32 * len(steps))(*steps), n_cu,
                           info, order, step, v, ctypes.byref(most))
    assert 0 <= n_bytes <= most.value
    names = ("n", "row_waves", "row_tiles", "per", "n_p", "p_tiles", "n_slots", "blocks", "most_chunks", "split", "heavy0", "heavy")
    return dict(zip(names, v), bytes=n_bytes)


NEVER, ALWAYS = (9, 0), (0, 0)


@pytest.mark.parametrize("split", [0, 256, 1024])
@pytest.mark.parametrize("C,T,heads,Tp,span,unspliced", [
    (48, 16, (32, 8, 128), 8192, (128, 8128), 24), (48, 16, (32, 8, 128), 8192, (0, 8192), 24), (48, 16, (32, 8, 128), 8192, (0, 8192), 1),
    (8, 4, (8, 2, 128), 32768, (0, 32768), 7), (8, 4, (8, 2, 128), 32768, (128, 32640), 7), (40, 12, (8, 4, 256), 4096, (0, 4096), 39)])
def test_shared_prompt_of_the_zero_donor(plan, C, T, heads, Tp, span, unspliced, split):
    """Spliced cells, which walk nothing of the span, do not take its chunks from the cells that walk all of it."""
    def of(donor_zero, lw):
        sh = sp.make_shape(C, 8, *heads, Tp, span, 1024, donor_zero, "bf16")
        return plan_of(plan, sh, sp.make_call(3, 0, 0, 0.1, split), sp.make_tree(T), lw, [7 * c for c in range(C)])
    alone = of(True, [NEVER] * C)
    some = of(True, [NEVER if c < unspliced else ALWAYS for c in range(C)])
    assert alone["n_p"] > 0 and some["n_p"] == alone["n_p"] and some["n_slots"] == alone["n_slots"]
    # nodes on both sides of the onset: no fewer chunks than for the unspliced ones
    inside = of(True, [(0, 7 * c + 1) if c < unspliced else ALWAYS for c in range(C)])
    assert inside["n_p"] >= alone["n_p"]
    # cells that are all spliced share what is left of the prompt, if anything
    none = of(True, [ALWAYS] * C)
    if span == (0, Tp):
        bare = plan_of(plan, sp.make_shape(C, 8, *heads, 0, (0, 0), 1024, True, "bf16"), sp.make_call(3, 0, 0, 0.1, split),
                       sp.make_tree(T), [ALWAYS] * C, [7 * c for c in range(C)])
        assert none == bare and none["n_p"] == 0
    else:
        assert none["n_p"] > 0 if split else none["n_p"] <= alone["n_p"]
    assert of(False, [NEVER] * C)["n_p"] == alone["n_p"]


def test_zero_donor_shares_the_prompt_like_unspliced_cells(plan):
    rng = random.Random(11)
    packed = 0
    for trial in range(2000):
        sh, call, tree, _, steps = draw(rng)
        sh.donor_kind = sp.SPLICE_DONOR_ZERO
        if rng.random() < 0.3:
            sh.span_lo, sh.span_hi = 0, sh.prompt_len
        active = [c for c in range(sh.n_cells) if steps[c] >= 0]
        # a spliced list, whose parts before and behind the span end in tiles of their own, is the shorter one from a span of a
        # tile on: ceil(x) + ceil(y) <= ceil(x + y) + 1
        low = sh.prompt_len + min((steps[c] for c in active), default=0) - call.window + 1 if call.window else 0
        if not active or sh.span_hi - max(sh.span_lo, low) < 64:
            continue
        lw = [rng.choice((NEVER, ALWAYS)) for _ in steps]
        lw[rng.choice(active)] = NEVER
        alone = plan_of(plan, sh, call, tree, [NEVER] * len(steps), steps)
        some = plan_of(plan, sh, call, tree, lw, steps)
        assert some["n_p"] == alone["n_p"], trial
        packed += alone["n_p"] > 0
    assert packed > 100


def test_shared_prompts_have_chunks(plan):
    """A call that leaves the prompt to shared items has some: else each cell's prompt would hang behind its last chunk."""
    rng = random.Random(13)
    for trial in range(2000):
        sh, call, tree, lw, steps = draw(rng)
        if rng.random() < 0.5:
            sh.donor_kind, sh.span_lo, sh.span_hi = sp.SPLICE_DONOR_ZERO, 0, sh.prompt_len
        p = plan_of(plan, sh, call, tree, lw, steps)
        if p["n"]:
            assert bool(p["split"]) == (p["n_slots"] > p["n"]), trial
