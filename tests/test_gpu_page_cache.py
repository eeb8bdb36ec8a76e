"""PageCache over the kernels: pools that run short, pages that cells share, passes that ask for rows without pages."""
import numpy as np
import pytest
import torch

import gpu_common as gc
import paper_2605_30574_amd as sp
from test_gpu_page_decoder import run, setup

pytestmark = pytest.mark.gpu


def test_shortage_freeing_retry_and_a_pass():
    """A cell that found no page gets one when another's come free, and its tokens are then seen."""
    w, m, lw, gpu, cpu = setup("blank-sink")
    C = lw.shape[0]
    rng = np.random.default_rng(5)
    gc.announce("pages, short")
    pages = gpu.make_pages(3, n_pages=2 * (-(-w.prompt_len // 64)) + C - 1)
    cache = pages.cache
    cache.reserve([64] * C)
    assert int(cache.missing) == 1 and cache.rows.tolist() == [64] * (C - 1) + [0]
    cache.fork([-1] + list(range(1, C)), [0] + [64] * (C - 2) + [0])
    cache.reserve([0] + [64] * (C - 1))
    assert int(cache.missing) == 0 and cache.rows.tolist() == [0] + [64] * (C - 1)
    tables = cache.tables.cpu().numpy()
    assert (tables[1:, 0] >= 0).all() and len(set(tables[1:, 0])) == C - 1 and (tables[0] == -1).all()
    steps = np.array([-1] + [0] * (C - 1), np.int32)
    run(gpu, cpu, pages, rng.integers(0, m.vocab, (C, 3)), steps, None, "after a shortage")
    run(gpu, cpu, pages, rng.integers(0, m.vocab, (C, 3)), np.where(steps >= 0, 3, -1).astype(np.int32), None, "after a shortage, on")


def test_a_copy_that_found_no_page():
    w, m, lw, gpu, _ = setup("blank-sink")
    C = lw.shape[0]
    gc.announce("pages, no copy")
    pages = gpu.make_pages(70, n_pages=2 * (-(-w.prompt_len // 64)) + 2)
    cache = pages.cache
    cache.reserve([70] + [0] * (C - 1))
    gpu.page_logits(torch.zeros(C, 70, dtype=torch.int64, device="cuda"), pages, np.array([0] + [-1] * (C - 1), np.int32))
    cache.fork([0] * C, [70] * C)
    assert int(cache.missing) == C - 1 and cache.rows.tolist() == [70] + [64] * (C - 1)
    with pytest.raises(ValueError):
        cache.reserve([70] * C)
    cache.fork([-1] + [1] * (C - 1), [0] + [64] * (C - 1), [0, 65] + [64] * (C - 2))
    assert int(cache.missing) == 0 and cache.rows.tolist() == [0, 65] + [64] * (C - 2)


def test_captured_fork():
    """A fork in a graph asks nothing of the device: each replay forks what the tables then hold."""
    w, m, lw, gpu, _ = setup("blank-sink")
    C = lw.shape[0]
    gc.announce("pages, captured fork")
    cache = gpu.make_pages(1).cache
    cache.reserve([70] * C)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        cache.fork([0] * C, [70] * C, [130] * C)
    assert cache.rows.tolist() == [130] * C
    for _ in range(3):
        graph.replay()
        torch.cuda.synchronize()
        tables, refs = cache.tables.cpu().numpy(), cache.refs.cpu().numpy()
        assert int(cache.missing) == 0 and len(set(tables[:, 0])) == 1 and len(set(tables[:, 1:].ravel())) == 2 * C
        held = cache._tables.cpu().numpy()
        assert (refs == np.bincount(held[held >= 0], minlength=len(refs))).all()


def test_a_pass_without_pages_is_refused():
    w, m, lw, gpu, _ = setup("blank-sink")
    C = lw.shape[0]
    gc.announce("pages, not reserved")
    pages = gpu.make_pages(2)
    tokens = torch.zeros(C, 2, dtype=torch.int64, device="cuda")
    with pytest.raises(ValueError):
        gpu.page_logits(tokens, pages, np.zeros(C, np.int32))
    pages.cache.reserve([2] * (C - 1) + [1])
    with pytest.raises(ValueError):
        gpu.page_logits(tokens, pages, np.zeros(C, np.int32))
    gpu.page_logits(tokens, pages, np.zeros(C, np.int32), [2] * (C - 1) + [1])
    for new in ([3] + [1] * (C - 1), [-1] + [1] * (C - 1)):
        with pytest.raises((ValueError, sp.SpliceError)):
            gpu.page_logits(tokens, pages, np.zeros(C, np.int32), new)
    torch.cuda.synchronize()


def test_rows_that_cells_share_are_not_written():
    """A step back into a shared page is refused; behind a fork to that row the pass writes the cells' own copies."""
    w, m, lw, gpu, cpu = setup("diff-G8")
    C = lw.shape[0]
    rng = np.random.default_rng(6)
    draw = lambda n: rng.integers(0, m.vocab, (C, n))  # noqa: E731
    gc.announce("pages, shared rows")
    pages = gpu.make_pages(130)
    cache = pages.cache
    cache.reserve([130] + [0] * (C - 1))
    trunk = np.array([0] + [-1] * (C - 1), np.int32)
    run(gpu, cpu, pages, draw(130), trunk, None, "trunk")
    cache.fork([0] * C, [130] * C)
    for x in (*cpu.gen_k, *cpu.gen_v):
        x[1:] = x[0]
    one, at = gpu.make_pages(1, cache=cache), np.array([127] + [-1] * (C - 1), np.int32)
    keep = torch.zeros(C, 1, dtype=torch.int32, device="cuda")
    for bad in (lambda: gpu.page_logits(torch.from_numpy(draw(1)).cuda(), one, at), lambda: cache.compact(at, keep),
                lambda: cache.compact(np.full(C, 100), keep)):
        with pytest.raises(ValueError):
            bad()
    run(gpu, cpu, one, draw(1), np.full(C, 129, np.int32), None, "the last row again")   # in the cells' own pages
    cache.fork(list(range(C)), [100] + [130] * (C - 1))
    cache.reserve([103] + [130] * (C - 1))
    cache.compact(np.where(np.arange(C) == 0, 100, -1), keep)
    steps = np.where(np.arange(C) == 0, 100, 129).astype(np.int32)
    run(gpu, cpu, gpu.make_pages(3, cache=cache), draw(3), steps, np.where(steps == 100, 3, 1).astype(np.int32), "back")


@pytest.mark.parametrize("name,prompts", [("zero-window5", 1), ("diff-G8", 2)])
def test_pages_by_default(name, prompts):
    """As many as the prompts and all cells can fill: a ZERO donor has none."""
    w, m, lw, gpu, _ = setup(name)
    C = lw.shape[0]
    gc.announce(f"pages by default {name}")
    cache = gpu.make_pages(1).cache
    assert cache.pools.shape[1] == prompts * -(-w.prompt_len // 64) + C * 3
    cache.reserve([140] * C)
    assert int(cache.missing) == 0 and int((cache.refs == 0).sum()) == 0
    cache.fork([1] * C, [100] * C, [140] * C)
    cache.fork(list(range(C)), [140] * C)
    assert int(cache.missing) == 0 and cache.rows.tolist() == [140] * C


def test_what_a_captured_fork_missed_is_noticed():
    w, m, lw, gpu, _ = setup("blank-sink")
    C = lw.shape[0]
    gc.announce("pages, captured shortage")
    cache = gpu.make_pages(1, n_pages=2 * (-(-w.prompt_len // 64)) + C).cache
    cache.reserve([64] + [0] * (C - 1))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        cache.reserve([128] * C)
    for _ in range(3):
        graph.replay()
        torch.cuda.synchronize()
        assert int(cache.missing) == C
    cache.fork([0] * C, [0] * C, [64] * C)
    assert int(cache.missing) == 0 and cache.rows.tolist() == [64] * C
    cache.reserve([64] * (C - 1) + [128])
    assert int(cache.missing) == 1 and cache.rows.tolist() == [64] * C
