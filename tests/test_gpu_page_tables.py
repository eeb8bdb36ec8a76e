"""splice_page_fork and splice_page_compact against the definitions, cell by cell."""
import numpy as np
import pytest
import torch

import page_reference as ref
import paper_2605_30574_amd as sp
from gpu_common import announce

pytestmark = pytest.mark.gpu
P = 64
up = lambda x, t=np.int32: torch.from_numpy(np.ascontiguousarray(np.asarray(x).astype(t))).cuda()  # noqa: E731


class Held:
    """Cells that hold pages of pools with random bytes."""

    def __init__(self, seed, rows, L=5, free=6, layers=3, Hkv=2, D=64, pinned=1, gap=0, shared=()):
        rng = np.random.default_rng(seed)
        self.rng, self.rows, self.C, self.L, self.layers, self.Hkv, self.D = rng, np.asarray(rows), len(rows), L, layers, Hkv, D
        used = sum(-(-r // P) for r in rows)
        self.n_pages = used + free
        order = rng.permutation(self.n_pages)
        self.tables, at = np.full((self.C, L), -1), 0
        for c, r in enumerate(rows):
            n = -(-r // P)
            self.tables[c, :n] = order[at:at + n]
            at += n
        for c, other, n in shared:      # the first n pages of a cell are another's
            self.tables[c, :n] = self.tables[other, :n]
        self.refs = np.bincount(self.tables[self.tables >= 0], minlength=self.n_pages)
        self.refs[order[used:used + pinned]] += 1
        self.bytes = Hkv * ref.head_bytes(D)
        self.mem = torch.from_numpy(rng.integers(0, 256, (layers, self.n_pages + gap, self.bytes), dtype=np.uint8)).cuda()
        self.pools = self.mem[:, :self.n_pages]
        self.shape = sp.make_shape(self.C, layers, Hkv, Hkv, D, 0, (0, 0), L * P, False, "bf16")

    def fork(self, parent, rows, want, stream=None):
        pages = sp.make_pages(self.n_pages, self.L)
        before = self.mem.cpu().numpy()
        tables, refs = up(self.tables), up(self.refs)
        new_t, new_r = torch.full_like(tables, 99), torch.full_like(refs, 99)
        missing, copied = torch.full((1,), 99, dtype=torch.int32, device="cuda"), torch.full((self.C, 2), 99, dtype=torch.int32, device="cuda")
        sp.splice_page_fork(self.shape, pages, parent, rows, want, tables, refs, new_t, new_r, missing, copied, self.pools, stream)
        torch.cuda.synchronize()
        t, r, m, cp = ref.fork(np.asarray(parent), np.asarray(rows), np.asarray(want), self.tables, self.refs, self.n_pages)
        assert (new_t.cpu().numpy() == t).all(), (new_t.cpu().numpy(), t)
        assert (new_r.cpu().numpy() == r).all()
        assert int(missing) == m
        assert (copied.cpu().numpy() == cp).all(), (copied.cpu().numpy(), cp)
        assert (tables.cpu().numpy() == self.tables).all() and (refs.cpu().numpy() == self.refs).all()
        for frm, to in cp:
            if frm >= 0:
                before[:, to] = before[:, frm]
        assert (self.mem.cpu().numpy() == before).all()
        assert not (cp[:, 1] >= 0).any() or (r[cp[cp[:, 1] >= 0, 1]] == 1).all()
        self.tables, self.refs, self.rows = t, r, np.asarray(rows)
        return m, cp


def test_fork_from_a_trunk_in_the_middle_of_a_page():
    announce("fork trunk")
    s = Held(1, [150, 0, 0, 0])
    m, cp = s.fork([0] * 4, [150, 150, 140, 128], [150, 200, 140, 129])
    assert m == 0 and (cp[0] == -1).all() and (cp[1] >= 0).all() and (cp[2] >= 0).all() and (cp[3] == -1).all()
    # and once more from a fork
    s.fork([0, 1, 1, 3], [150, 200, 131, 129], [151, 201, 132, 129])


def test_free_keep_fewer_and_grow():
    announce("fork free")
    s = Held(2, [320, 65, 64, 1, 0])
    s.fork([-1, 1, 2, 3, 4], [0, 60, 64, 1, 0], [0, 60, 65, 320, 1])
    s.fork([-1] * 5, [0] * 5, [0] * 5)
    assert s.refs.sum() == 1      # the page that somebody else holds


def test_beams_swap_and_gather():
    announce("fork beams")
    s = Held(3, [100, 130, 64, 300], free=12)
    s.fork([1, 0, 1, 1], [130, 100, 130, 65], [140, 101, 130, 128])
    s.fork([3, 3, 3, 3], [64, 64, 65, 60], [65, 64, 65, 61])


def test_nobody_keeps_a_page_that_others_hold_whole():
    announce("fork held whole")
    s = Held(4, [128, 0, 0], shared=())
    m, cp = s.fork([0, 0, 0], [128, 70, 70], [128, 70, 70])
    assert (cp[0] == -1).all() and (cp[1:] >= 0).all()
    s = Held(5, [70, 0], pinned=0)
    s.refs[s.tables[0, 1]] += 1   # held by somebody outside of the tables
    m, cp = s.fork([0, 0], [70, 70], [70, 70])
    assert (cp >= 0).all()


@pytest.mark.parametrize("free", [0, 1, 2, 3])
def test_too_few_pages(free):
    announce(f"fork short {free}")
    s = Held(6, [150, 0, 0], free=free, pinned=0)
    m, _ = s.fork([0, 0, 0], [150, 150, 150], [150, 200, 300])
    assert m == 5 - free


def test_absent_entries_and_one_page():
    announce("fork absent")
    s = Held(7, [150, 10])
    s.tables[0, 1], s.tables[1, 3] = -7, s.n_pages + 5
    s.refs = np.bincount(s.tables[(s.tables >= 0) & (s.tables < s.n_pages)], minlength=s.n_pages)
    s.fork([0, 0], [150, 100], [150, 130])
    s = Held(8, [0], L=1, free=1, pinned=0, layers=1)
    s.fork([0], [0], [64])
    s.fork([0], [64], [64])


@pytest.mark.parametrize("seed", range(6))
def test_random_forks(seed):
    announce(f"fork random {seed}")
    rng = np.random.default_rng(seed)
    C = int(rng.choice([1, 3, 17, 130, 256]))
    s = Held(seed, rng.integers(0, 321, C), free=int(rng.choice([3, C, 6 * C])), layers=2, Hkv=1, gap=seed % 2)
    for _ in range(4):
        parent = np.where(rng.random(C) < 0.2, np.arange(C), rng.integers(-1, C, C))
        rows = np.array([0 if p < 0 else rng.integers(0, s.rows[p] + 1) for p in parent])
        rows = np.where(rng.random(C) < 0.3, rows // P * P, rows)
        want = np.minimum(320, rows + rng.integers(0, 100, C))
        s.fork(parent.tolist(), rows.tolist(), want.tolist())


def test_many_pages():
    """More free pages than one pass over the counts sees, and free ones far behind."""
    announce("fork many pages")
    s = Held(9, [320] * 40, L=5, free=5000, layers=1, Hkv=1)
    s.refs[:4000] += 1
    s.fork(list(range(40)), [320 - 7 * c for c in range(40)], [320] * 40)


def around(free, layers=1):
    """Three cells in a pool of so many pages more than they hold."""
    return Held(28, [150, 320, 70], free=free, layers=layers, Hkv=1)


@pytest.mark.parametrize("n_pages", [12287, 12288, 12289, 16384, 30011])
def test_pools_with_more_pages_than_counts_fit_in_lds(n_pages):
    """Counts in LDS up to 12288 pages, in memory above: trunk, beams, cells that give back, few free pages and those far behind."""
    announce(f"fork of {n_pages} pages")
    s = around(n_pages - 10)
    assert s.n_pages == n_pages
    m, cp = s.fork([0, 0, 0], [150, 140, 128], [200, 320, 130])
    assert m == 0 and (cp[0] == -1).all() and (cp[1] >= 0).all()
    s.fork([1, 2, 1], [300, 65, 70], [300, 100, 71])
    s.fork([-1, 1, 2], [0, 60, 64], [320, 60, 64])
    s.fork([0, 1, 0], [320, 60, 256], [320, 320, 256])
    # none free but the last three
    s.fork([0, -1, -1], [64, 0, 0], [64, 0, 0])
    taken = np.flatnonzero(s.refs == 0)[:-3]
    s.refs[taken] += 1
    m, cp = s.fork([0, 0, 0], [64, 64, 40], [128, 320, 40])
    assert m == 3 and (cp == -1).all() and s.refs.min() > 0      # the copy of the last cell's page among them
    # and those far behind the first ones that are not
    s.refs[taken[-200:]] -= 1
    m, cp = s.fork([0, 0, 0], [128, 100, 40], [320, 320, 320])
    assert m == 0 and (cp[1:] >= 0).all()


@pytest.mark.parametrize("seed", range(4))
def test_random_forks_with_counts_in_memory(seed):
    announce(f"fork random, many pages {seed}")
    rng = np.random.default_rng(seed)
    C = int(rng.choice([3, 130, 256]))
    s = Held(seed, rng.integers(0, 321, C), free=13000, layers=2, Hkv=1)
    s.refs[np.flatnonzero(s.refs == 0)[:-int(rng.choice([1, C]))]] += 1
    for _ in range(3):
        parent = np.where(rng.random(C) < 0.2, np.arange(C), rng.integers(-1, C, C))
        rows = np.array([0 if p < 0 else rng.integers(0, s.rows[p] + 1) for p in parent])
        rows = np.where(rng.random(C) < 0.3, rows // P * P, rows)
        s.fork(parent.tolist(), rows.tolist(), np.minimum(320, rows + rng.integers(0, 200, C)).tolist())


def test_replayed_fork_with_counts_in_memory():
    announce("fork graph, many pages")
    s = around(13000)
    bufs = [up(s.tables), up(s.refs)]
    outs = [torch.zeros_like(bufs[0]), torch.zeros_like(bufs[1]), torch.zeros(1, dtype=torch.int32, device="cuda"),
            torch.zeros(3, 2, dtype=torch.int32, device="cuda")]
    args = [0, 0, 2], [150, 140, 70], [150, 200, 130]
    call = lambda: sp.splice_page_fork(s.shape, sp.make_pages(s.n_pages, s.L), *args, *bufs, *outs, s.pools)  # noqa: E731
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for i in range(4):
        refs = s.refs.copy()
        refs[np.flatnonzero(refs == 0)[:50 * i]] += 1         # other pages are free
        bufs[1].copy_(up(refs))
        for x in outs:
            x.fill_(-5)
        graph.replay()
        torch.cuda.synchronize()
        for x, y in zip(outs, ref.fork(*(np.asarray(x) for x in args), s.tables, refs, s.n_pages)):
            assert (x.cpu().numpy().reshape(np.shape(y)) == y).all(), i


def test_fork_graph_and_stream():
    announce("fork graph")
    s = Held(10, [150, 0, 70], free=9)
    pages = sp.make_pages(s.n_pages, s.L)
    bufs = [up(s.tables), up(s.refs)]
    outs = [torch.zeros_like(bufs[0]), torch.zeros_like(bufs[1]), torch.zeros(1, dtype=torch.int32, device="cuda"),
            torch.zeros(3, 2, dtype=torch.int32, device="cuda")]
    call = lambda: sp.splice_page_fork(s.shape, pages, [0, 0, 2], [150, 140, 70], [150, 200, 130], *bufs, *outs, s.pools)  # noqa: E731
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for i in range(4):
        s.pools.copy_(torch.randint(0, 256, s.pools.shape, dtype=torch.uint8, device="cuda"))
        before = s.pools.clone()
        for x in outs:
            x.fill_(-5)
        graph.replay()
        torch.cuda.synchronize()
        got = [x.clone() for x in outs] + [s.pools.clone()]
        s.pools.copy_(before)
        call()
        torch.cuda.synchronize()
        for x, y in zip(got, outs + [s.pools]):
            assert torch.equal(x, y), i
    side = torch.cuda.Stream()
    Held(11, [150, 0], free=9).fork([0, 0], [150, 150], [150, 150], side)


# ---------------------------------------------------------------- compact

def compact(s, base, keep, T=None, cap=None, stream=None):
    T = T or max(len(k) for k in keep)
    lists = np.full((s.C, T), -1, np.int64)
    for c, k in enumerate(keep):
        lists[c, :len(k)] = k
    cap = cap or s.L * P
    shape = sp.make_shape(s.C, s.layers, s.Hkv, s.Hkv, s.D, 0, (0, 0), cap, False, "bf16")
    before, mem = s.mem.cpu().numpy(), None
    sp.splice_page_compact(shape, sp.make_pages(s.n_pages, s.L, T), base, up(lists), up(s.tables), s.pools, stream)
    torch.cuda.synchronize()
    mem = s.mem.cpu().numpy()
    want = before.copy()
    at = lambda r: [np.broadcast_to(x, s.D) for x in ref.places(r % P, np.arange(s.D), s.D)]  # noqa: E731
    ok = lambda p: 0 <= p < s.n_pages  # noqa: E731
    for c in range(s.C):
        if base[c] < 0:
            continue
        for i, k in enumerate(ref.kept(lists[c], cap - base[c])):
            frm, to = base[c] + k, base[c] + i
            p, q = s.tables[c, frm // P], s.tables[c, to // P]
            if not (ok(p) and ok(q)):
                continue
            for h in range(s.Hkv):
                off = h * ref.head_bytes(s.D)
                for x, y in zip(at(frm), at(to)):
                    want[:, q, off + y] = before[:, p, off + x]
    assert (mem == want).all(), f"{(mem != want).sum()} bytes off, first at {np.argwhere(mem != want)[0]}"


@pytest.mark.parametrize("D,Hkv", [(64, 1), (64, 3), (128, 2), (256, 2)])
def test_accepted_tokens(D, Hkv):
    announce(f"compact accepted {D} {Hkv}")
    s = Held(20, [320] * 6, Hkv=Hkv, D=D)
    compact(s, [0, 60, 64, 200, -1, 313], [[0, 1, 2], [1, 3, 4, 6], [6], [], [0, 2], [0, 3, 6]], T=7)


@pytest.mark.parametrize("share", [0.02, 0.3, 0.7, 0.97, 1.0])
@pytest.mark.parametrize("D", [64, 128, 256])
def test_rows_that_an_eviction_leaves(share, D):
    announce(f"compact evict {share} {D}")
    s = Held(21, [640] * 4, L=10, layers=2, D=D)
    rng = np.random.default_rng(int(100 * share))
    base = [0, 1, 63, 130]
    compact(s, base, [np.flatnonzero(rng.random(640 - b) < share) for b in base], T=640)


def test_whole_pages_dropped_and_kept():
    announce("compact pages")
    s = Held(22, [640] * 4, L=10, layers=1)
    compact(s, [0, 0, 32, 0], [list(range(64, 128)) + list(range(320, 448)), list(range(448)) + [639], list(range(64, 256)), [639]], T=449)


def test_lists_end():
    announce("compact lists")
    s = Held(23, [320] * 6, layers=1)
    compact(s, [0, 0, 0, 10, 300, 320], [[3, 5, 5, 9], [3, 5, 4, 9], [3, -1, 7, 9], [3, 309, 310, 311], [1, 19, 20, 21], [0, 1, 2, 3]], T=4)
    s = Held(24, [320] * 2, layers=1)
    compact(s, [0, 5], [[1, 2**31 - 1, 7], [2**31 - 4, 2**31 - 3, 2**31 - 2]], T=3)
    s = Held(25, [320] * 2, layers=1)
    compact(s, [0, 100], [[1, 150, 199, 200], [1, 99, 100, 101]], T=4, cap=200)


def test_compact_absent_pages_and_strided_layers():
    announce("compact absent")
    s = Held(26, [320] * 3, layers=3, gap=2)
    s.tables[0, 1], s.tables[1, 0], s.tables[2, 4] = -1, s.n_pages, 2**31 - 1
    rng = np.random.default_rng(3)
    compact(s, [0, 0, 0], [np.flatnonzero(rng.random(320) < 0.5) for _ in range(3)], T=320)


def test_many_cells_and_another_stream():
    announce("compact many")
    rng = np.random.default_rng(4)
    s = Held(27, [128] * 200, L=2, layers=1, Hkv=1)
    compact(s, rng.integers(-1, 120, 200).tolist(), [np.flatnonzero(rng.random(8) < 0.5) for _ in range(200)], T=8, stream=torch.cuda.Stream())
