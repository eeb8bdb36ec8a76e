"""The host-side plan of splice_page_attn (csrc/page_plan.hpp), compiled here for the CPU: every row has its tiles, every list its
parts, and the workspace that is asked for holds every partial result."""
import ctypes
import os
import random
import subprocess

import pytest

import paper_2605_30574_amd as sp
from paper_2605_30574_amd import pages as PG

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SRC = r"""
#include "page_plan.hpp"
using namespace splice;
extern "C" {
int prepare(const splice_shape *sh, const splice_call *call, const splice_pages *pg, const int32_t *cells, int n, int units, int64_t *v) {
    if (validate_pages(sh, pg) != SPLICE_OK) return -1;
    PageCell c[SPLICE_MAX_CELLS];
    for (int i = 0; i < n; ++i) c[i] = {cells[4 * i], cells[4 * i + 1], cells[4 * i + 2], cells[4 * i + 3]};
    const PagePlan p = page_plan(*sh, *call, *pg, c, n, units);
    const int64_t w[] = {p.own, p.shared, p.own_rows, p.own_tiles, p.own_each, p.own_per, p.own_parts, p.rows_u, p.rows_s, p.tiles_u,
                         p.tiles_s, p.prompt_per, p.prompt_parts, p.parts, p.blocks, p.bytes,
                         page_most_parts(*sh, *pg) * page_part_bytes(*sh, *pg), page_part_bytes(*sh, *pg)};
    for (int i = 0; i < 18; ++i) v[i] = w[i];
    return 0;
}
}
"""
NAMES = ("own", "shared", "own_rows", "own_tiles", "own_each", "own_per", "own_parts", "rows_u", "rows_s", "tiles_u", "tiles_s",
         "prompt_per", "prompt_parts", "parts", "blocks", "bytes", "most", "part_bytes")


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    d = tmp_path_factory.mktemp("page_plan")
    src, so = d / "plan.cpp", d / "plan.so"
    src.write_text(SRC)
    subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-Wall", "-Werror", "-D_GLIBCXX_ASSERTIONS", "-fsanitize=undefined",
                    "-fno-sanitize-recover", "-I", os.path.join(ROOT, "include"), "-I", os.path.join(ROOT, "paper_2605_30574_amd", "csrc"),
                    "-o", str(so), str(src)], check=True)
    lib = ctypes.CDLL(str(so))

    def run(sh, call, pages, cells, units=256):
        flat = [x for c in cells for x in c]
        v = (ctypes.c_int64 * 18)()
        assert lib.prepare(ctypes.byref(sh), ctypes.byref(call), ctypes.byref(pages), (ctypes.c_int32 * len(flat))(*flat), len(cells), units, v) == 0
        return dict(zip(NAMES, v))
    return run


def up(a, b):
    return -(-a // b)


def draw(rng):
    log = lambda lo, hi: int(round(lo * (hi / lo) ** rng.random()))  # noqa: E731
    C, T = log(1, 256), log(1, 32768) if rng.random() < 0.3 else log(1, 40)
    Hkv, G, D = rng.choice((1, 2, 4, 8, 32)), rng.choice((1, 2, 4, 8)), rng.choice((64, 128, 256))
    Tp, cap = rng.choice((0, log(1, 200000))), T + log(1, 100000)
    a = rng.randint(0, Tp)
    sh = sp.make_shape(C, 8, Hkv * G, Hkv, D, Tp, (a, rng.randint(a, Tp)), cap, rng.random() < 0.3, "bf16")
    call = sp.make_call(3, 0, rng.choice((0, 0, log(1, 5000))), 0.1, rng.choice((0, 0, 0, 64, 256, 65536)))
    cells = []
    for c in range(C):
        n = rng.choice((T, rng.randint(1, T)))
        cells.append((c, rng.randint(0, cap - n), n, rng.choice((0, n, rng.randint(0, n)))))
    return sh, call, sp.make_pages(100, up(cap, 64), T), cells, G


def test_plans(plan):
    rng = random.Random(7)
    shared = split = wide = 0
    for trial in range(1500):
        sh, call, pages, cells, G = draw(rng)
        p = plan(sh, call, pages, cells, rng.choice((256, 304, 1)))
        most = max(c[2] for c in cells) * G
        assert p["own_rows"] == {0: 128 if sh.head_dim <= 128 else 64, 1: 16, 2: 32}[p["own"]] and (p["own"] or most > 64)
        assert not (p["shared"] and p["own"] == 0) and (p["own"] < 2 or sh.head_dim <= 128)
        tiles = [up(s * G, p["own_rows"]) + up((n - s) * G, p["own_rows"]) for _, _, n, s in cells]
        if p["shared"]:
            tiles = [up(n * G, p["own_rows"]) for _, _, n, _ in cells]
            assert sh.prompt_len > 0
            assert p["rows_u"] == sum(s for _, _, _, s in cells) * G and p["rows_u"] + p["rows_s"] == sum(n for _, _, n, _ in cells) * G
            rows = 128 if sh.head_dim <= 128 else 64
            assert p["tiles_u"] == up(p["rows_u"], rows) and p["tiles_s"] == up(p["rows_s"], rows)
            assert p["prompt_parts"] >= 1 and p["prompt_per"] >= 1
            # at most two pages more than the slots in view fill: the span's ends
            seen = min(sh.prompt_len, call.window) if call.window else sh.prompt_len
            assert p["prompt_per"] * p["prompt_parts"] >= up(seen, 64)
        else:
            assert p["prompt_parts"] == 0 and p["tiles_u"] == p["tiles_s"] == 0
        assert p["own_tiles"] == sum(tiles) and p["own_each"] == (tiles[0] if len(set(tiles)) == 1 else 0)
        assert p["own_parts"] >= 1 and p["own_per"] >= 1
        assert p["parts"] == p["own_parts"] + p["prompt_parts"] <= 64
        assert p["blocks"] == sh.n_kv_heads * (p["own_tiles"] * p["own_parts"] + (p["tiles_u"] + p["tiles_s"]) * p["prompt_parts"])
        assert p["bytes"] == (p["parts"] * p["part_bytes"] if p["parts"] > 1 else 0) <= p["most"]
        assert p["part_bytes"] >= sh.n_cells * pages.n_tokens * sh.n_q_heads * (sh.head_dim + 2) * 4 and p["part_bytes"] % 256 == 0
        shared += p["shared"]
        split += p["own_parts"] > 1
        wide += p["own"] == 0
    assert shared > 50 and split > 100 and wide > 100


def test_what_the_plan_is_for(plan):
    """One small call is one launch; a long list is cut; a prompt that many cells walk is shared, a short one is not."""
    one = plan(sp.make_shape(4, 4, 4, 2, 64, 32, (4, 28), 100, True, "bf16"), sp.make_call(1, 0, 0, 0.1), sp.make_pages(9, 2, 1),
               [(c, 50, 1, 0) for c in range(4)])
    assert one["parts"] == 1 and not one["shared"]
    long = plan(sp.make_shape(1, 4, 32, 8, 128, 131072, (4, 28), 100, True, "bf16"), sp.make_call(1, 0, 0, 0.1), sp.make_pages(9, 2, 1),
                [(0, 50, 1, 0)])
    assert long["own_parts"] > 8
    many = [(c, 500, 1, c % 2) for c in range(128)]
    shape = lambda Tp: sp.make_shape(128, 4, 32, 8, 128, Tp, (4, 28), 1000, False, "bf16")  # noqa: E731
    assert plan(shape(8192), sp.make_call(1, 0, 0, 0.1), sp.make_pages(9, 16, 1), many)["shared"]
    assert not plan(shape(64), sp.make_call(1, 0, 0, 0.1), sp.make_pages(9, 16, 1), many)["shared"]
    prompt = plan(sp.make_shape(1, 4, 32, 8, 128, 0, (0, 0), 4096, False, "bf16"), sp.make_call(1, 0, 0, 0.1), sp.make_pages(9, 64, 4096),
                  [(0, 0, 4096, 0)])
    assert prompt["own"] == 0 and prompt["parts"] == 1


def test_shapes_of_the_gpu_tests_share_their_prompts(plan):
    from page_common import SHARED, shared_case
    for (donor, window), cases in SHARED.items():
        own = set()
        for case in cases:
            c = shared_case(*case)
            T = c["T"]
            cells = [(i, s, T, T if L > 1 else min(T, max(0, W - s))) for i, (s, (L, W)) in enumerate(zip(c["steps"], c["LW"]))]
            sh = sp.make_shape(c["C"], 4, c["Hq"], c["Hkv"], c["D"], c["Tp"], c["span"], c["cap"], donor == "zero", "bf16")
            p = plan(sh, sp.make_call(1, 0, window, 0.1), sp.make_pages(999, 2, T), cells)
            assert p["shared"] and p["prompt_parts"] > 1 and p["rows_u"] and p["rows_s"], (donor, window, case)
            own.add((c["D"], p["own"]))
        # every kernel that has such tiles
        assert own >= {(64, 1), (128, 1), (128, 2), (256, 1)} and (window or (64, 2) in own), own


def test_ragged_shapes_of_the_gpu_tests_share_their_prompts(plan):
    from page_common import RAGGED, ragged_case
    for case in RAGGED:
        c = ragged_case(*case)
        cells = [(i, int(s), int(n), int(n) if L > 1 else min(int(n), max(0, W - int(s))))
                 for i, (s, n, (L, W)) in enumerate(zip(c["steps"], c["new"], c["LW"])) if s >= 0 and n > 0]
        assert len(cells) < c["C"] and (c["T"] == 1 or len({n for _, _, n, _ in cells}) > 1)
        sh = sp.make_shape(c["C"], 4, c["Hq"], c["Hkv"], c["D"], c["Tp"], c["span"], c["cap"], c["donor"] == "zero", "bf16")
        p = plan(sh, sp.make_call(1, 0, c["window"], 0.1), sp.make_pages(999, 2, c["T"]), cells)
        assert p["shared"] and p["prompt_parts"] > 1 and p["rows_u"] and p["rows_s"], (case, p)
