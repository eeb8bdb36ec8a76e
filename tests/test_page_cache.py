"""PageCache on the CPU: what it keeps of its cells' pages, with tests/page_reference.py's fork in the place of the kernel."""
from types import MethodType, SimpleNamespace

import numpy as np
import pytest
import torch

import page_reference as ref
import paper_2605_30574_amd as sp
from paper_2605_30574_amd import pages as PG
from paper_2605_30574_amd.decode import SweepDecoder

P = 64


def fork(shape, pages, parent, rows, want, tables, refs, new_tables, new_refs, missing, copied, pools, stream=None):
    got = ref.fork(*(np.asarray(x) for x in (parent, rows, want)), tables.numpy(), refs.numpy(), pages.n_pages)
    for out, x in zip((new_tables, new_refs, missing, copied), got):
        out.copy_(torch.from_numpy(np.asarray(x, dtype=np.int32).reshape(out.shape)))
    for frm, to in got[3]:
        if frm >= 0:
            pools[:, to] = pools[:, frm]


@pytest.fixture
def cache(monkeypatch):
    monkeypatch.setattr(PG, "splice_page_fork", fork)
    return lambda C, n_pages, capacity=320, Tp=0: sp.PageCache(C, 1, 2, 1, 64, Tp, (0, 0), capacity, n_pages, device="cpu")


def held(c):
    """Rows of every cell up to its first absent page."""
    there = np.cumprod(c.tables.numpy() >= 0, axis=1).sum(1)
    return (there * P).tolist()


def test_a_shortage_is_made_good_when_pages_come_free(cache):
    c = cache(2, 1)
    c.reserve([64, 64])
    assert int(c.missing) == 1 and c.rows.tolist() == [64, 0]
    c.reserve([64, 64])
    assert int(c.missing) == 1 and c.rows.tolist() == [64, 0]      # and is told again
    c.fork([-1, 1], [0, 0], [0, 0])
    c.reserve([0, 64])
    assert int(c.missing) == 0 and c.rows.tolist() == [0, 64] == held(c)


def test_no_hole_is_left_below_rows_that_are_given_later(cache):
    c = cache(2, 2)
    c.reserve([128, 64])
    assert int(c.missing) == 1 and c.rows.tolist() == [128, 0]
    c.fork([0, 1], [64, 0], [64, 128])
    assert int(c.missing) == 1 and c.rows.tolist() == [64, 64] == held(c)
    c.fork([-1, 1], [0, 64], [0, 128])
    assert int(c.missing) == 0 and c.rows.tolist() == [0, 128] == held(c)


def test_a_part_of_what_is_wanted(cache):
    c = cache(2, 4)
    c.reserve([130, 130])
    assert int(c.missing) == 2 and c.rows.tolist() == [130, 64] and held(c) == [192, 64]
    with pytest.raises(ValueError):
        c.fork([1, 1], [65, 64])                                   # cell 1 has no such row


def test_rows_lost_with_the_page_that_was_to_be_copied(cache):
    """A fork in the middle of a page, and no page for the copy: the cell has its whole pages, and is given none behind
    them in the place of the rows that it lost until a fork says what it goes on from."""
    c = cache(2, 3)
    c.reserve([70, 0])
    c.refs[2] += 1                                                 # the third page is somebody else's
    c.fork([0, 0], [70, 70], [80, 80])
    assert int(c.missing) == 1 and c.rows.tolist() == [80, 64]
    c.refs[2] -= 1
    with pytest.raises(ValueError):
        c.reserve([80, 80])
    c.reserve([80, 64])                                            # as it is
    with pytest.raises(ValueError):
        c.reserve([80, 128])
    c.fork([0, 0], [70, 70], [80, 80])                             # from the same rows once more
    assert int(c.missing) == 0 and c.rows.tolist() == [80, 80]
    c.reserve([100, 100])
    c.fork([0, 0], [70, 70], [80, 80])
    assert c.rows.tolist() == [80, 80]


def test_a_cell_that_lost_rows_may_go_on_from_those_it_has(cache):
    c = cache(2, 2)
    c.reserve([70, 0])
    c.fork([0, 0], [70, 70])
    assert int(c.missing) == 1 and c.rows.tolist() == [70, 64]
    c.fork([-1, 1], [0, 64], [0, 70])
    assert int(c.missing) == 0 and c.rows.tolist() == [0, 70]
    c.reserve([0, 128])
    assert int(c.missing) == 0 and c.rows.tolist() == [0, 128]


@pytest.mark.parametrize("seed", range(8))
def test_rows_are_those_that_have_pages(cache, seed):
    rng = np.random.default_rng(seed)
    C = int(rng.choice([1, 3, 9]))
    c = cache(C, 4 + int(rng.integers(1, 3 * C + 3)), Tp=70)           # four of them the prompts'
    for _ in range(30):
        if rng.random() < 0.5:
            want = rng.integers(0, 321, C)
            try:
                c.reserve(want)
            except ValueError:
                c.fork(np.arange(C), c.rows, c.rows)
                continue
        else:
            parent = rng.integers(-1, C, C)
            rows = np.array([0 if p < 0 else rng.integers(0, c.rows[p] + 1) for p in parent])
            want = np.minimum(320, rows + rng.integers(0, 130, C))
            c.fork(parent, rows, want)
        assert (c.rows <= want).all() and (c.rows <= held(c)).all()
        short = c.rows < want
        assert short.any() == (int(c.missing) > 0) and (c.rows[short] == np.array(held(c))[short]).all()
        assert (c.tables.numpy()[np.arange(c.table_len) >= -(-c.rows[:, None] // P)] == -1).all()


def ask(c, n, steps, new=None):
    """page_logits up to where the host has looked the call over: it stops at the weights, of which there are none."""
    d = SimpleNamespace(C=c.n_cells, w=SimpleNamespace(n_q_heads=2, n_kv_heads=1, head_dim=64), wt={})
    d.positions = MethodType(SweepDecoder.positions, d)
    pages = SimpleNamespace(cache=c, spec=c.pages(n))
    with pytest.raises(KeyError, match="embed"):
        SweepDecoder.page_logits(d, torch.zeros(c.n_cells, n, dtype=torch.int64), pages, np.asarray(steps, np.int32), new)


def test_a_pass_over_rows_without_pages_is_refused(cache):
    c = cache(3, 9)
    c.reserve([64, 10, 0])
    ask(c, 4, [60, 6, -1])
    ask(c, 4, [60, 6, 0], [4, 4, 0])
    ask(c, 4, [64, 8, -5], [0, 2, 4])
    for steps, new in (([61, 6, -1], None), ([60, 7, -1], None), ([60, 6, 0], None), ([60, 8, -1], [4, 3, 0]), ([0, 0, 0], [0, 0, 1]),
                       ([2**31 - 1, 0, -1], None), ([0, 0, -1], [1, 1])):
        with pytest.raises(ValueError):
            ask(c, 4, steps, new)
    short = cache(2, 1)
    short.reserve([64, 64])
    ask(short, 1, [63, -1])
    with pytest.raises(ValueError):
        ask(short, 1, [0, 0])


def shared_rows(c):
    """Of every cell, the rows up to the last page that another cell's table names too."""
    t = c.tables.numpy()
    pages, number = np.unique(t[t >= 0], return_counts=True)
    return [max([(j + 1) * P for j, p in enumerate(row) if p in pages[number > 1]], default=0) for row in t]


@pytest.mark.parametrize("seed", range(10))
def test_rows_of_pages_that_other_cells_have_are_not_written(cache, monkeypatch, seed):
    """compact and a pass from a row on that lies in another cell's page too are refused, all others are not."""
    calls = []
    monkeypatch.setattr(PG, "splice_page_compact", lambda *a: calls.append(a))
    rng = np.random.default_rng(100 + seed)
    C = int(rng.choice([1, 2, 5, 12]))
    c = cache(C, int(rng.choice([2 * C + 1, 5 * C])))
    refused = 0
    for _ in range(25):
        if rng.random() < 0.4:
            want = np.minimum(rng.integers(0, 321, C), np.where(c._lost, c.rows, 320))
            c.reserve(want)
        else:
            parent = np.where(rng.random(C) < 0.3, np.arange(C), rng.integers(-1, C, C))
            rows = np.array([0 if p < 0 else (c.rows[p] if rng.random() < 0.4 else rng.integers(0, c.rows[p] + 1)) for p in parent])
            rows = np.where(rng.random(C) < 0.4, rows // P * P, rows)
            c.fork(parent, rows, np.minimum(320, rows + rng.integers(0, 130, C)))
        shared = shared_rows(c)
        for cell in range(C):
            for step in {0, 1, 63, 64, max(shared[cell] - 1, 0), shared[cell], int(c.rows[cell])}:
                steps = np.full(C, -1)
                steps[cell] = step
                keep = torch.zeros(C, 4, dtype=torch.int32)
                if step < shared[cell]:
                    refused += 1
                    with pytest.raises(ValueError):
                        c.compact(steps, keep)
                else:
                    c.compact(steps, keep)
                    assert calls.pop()[2] is steps and not calls
                if step < c.rows[cell]:
                    if step < shared[cell]:
                        with pytest.raises(ValueError):
                            ask(c, 1, steps)
                    else:
                        ask(c, 1, steps)
    assert refused or C == 1


def test_pages_become_a_cells_own_again(cache):
    c = cache(2, 8)
    c.reserve([130, 0])
    c.fork([0, 0], [130, 128], [130, 140])
    with pytest.raises(ValueError):
        ask(c, 1, [127, -1])
    ask(c, 1, [128, 128])
    with pytest.raises(ValueError):
        c.compact([-1, 100], torch.zeros(2, 4, dtype=torch.int32))
    c.fork([0, 1], [130, 100], [130, 101])            # cell 1 drops rows 100 ..: the page of the others is copied
    ask(c, 1, [128, 100])
    ask(c, 1, [64, 64])
    with pytest.raises(ValueError):
        ask(c, 1, [63, -1])
    c.fork([0, -1], [130, 0], [130, 0])               # cell 1 gives its pages back
    ask(c, 1, [0, -1])


def test_a_step_that_needs_no_page_does_not_wait(cache, monkeypatch):
    """reserve within a cell's own last page reads nothing back; a copy that it may need is read."""
    c = cache(2, 8)
    c.reserve([65, 65])
    read = []
    monkeypatch.setattr(torch.Tensor, "__int__", lambda t: read.append(t) or 0)
    for n in (66, 67, 128):
        c.reserve([n, n])
    assert not read
    c.reserve([129, 128])
    assert len(read) == 1
    c.fork([0, 0], [128, 128])                        # whole pages alone
    assert len(read) == 1
    c.reserve([100, 128])                             # the end of a page that cell 1 has too
    assert len(read) == 2
    c.fork([0, 0], [70, 0])                           # of a page that is cell 0's alone
    assert len(read) == 2
    c.fork([0, 0], [70, 70])
    assert len(read) == 3


def test_a_shortage_that_was_not_waited_for_is_noticed_behind_the_next_wait(cache):
    """A page that somebody holds by its count is copied by a call that the host does not wait for."""
    c = cache(2, 3)
    c.reserve([70, 10])
    c.refs += 1                                       # all pages
    c.reserve([80, 10])
    assert int(c.missing) == 2 and c.rows.tolist() == [80, 10]
    c.refs -= 1
    c.reserve([140, 10])                              # asks for a page and is waited for
    assert c.rows.tolist() == [64, 0]
    with pytest.raises(ValueError):
        c.reserve([140, 0])
    with pytest.raises(ValueError):
        c.reserve([64, 10])
    c.fork([0, -1], [64, 0], [140, 10])
    assert int(c.missing) == 1 and c.rows.tolist() == [140, 0]


def test_no_cells(cache):
    c = cache(0, 2, Tp=60)
    c.fork([], [], [])
    c.reserve([])
    assert int(c.missing) == 0 and c.rows.size == 0 and c.refs.tolist() == [1, 1]
