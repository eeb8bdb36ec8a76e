"""Python binding of include/splice_pages.h: K and V in 4 bits, in pages of 64 tokens that cells share.

A layer's pool is a uint8 tensor [n_pages][splice_page_bytes(shape)]; a cell's rows lie in the pages that its row of a table
(int32 [C][table_len] on the device) names.  ``splice_page_append`` writes new tokens, ``splice_page_attn`` attends,
``splice_page_fork`` says who holds which pages next, ``splice_page_compact`` moves the rows that stay together, and
``splice_page_read`` reads rows back.  ``PageCache`` keeps the pools, tables and counts of a sweep, and
``decode.SweepDecoder.page_logits`` runs a pass over them.

As in ``splice``, functions have the C names, marshal arguments only and check every tensor's device, dtype, layout and size
before calling into C; a negative status raises ``SpliceError``.  The kernels run on the current device: tensors of another one
are refused.
"""
from __future__ import annotations

import ctypes
from typing import Optional, Tuple

import numpy as np

from . import splice as S
from . import tree as T

SPLICE_PAGE_ROWS, SPLICE_MAX_PAGE_TOKENS = 64, 32768

EXPORTS = ("splice_page_bytes", "splice_page_append", "splice_page_read", "splice_page_attn_workspace_bytes",
           "splice_page_attn", "splice_page_fork", "splice_page_compact")


class SplicePages(ctypes.Structure):
    _fields_ = [("n_pages", ctypes.c_int32), ("table_len", ctypes.c_int32), ("n_tokens", ctypes.c_int32)]


_declared = None


def _library():
    """The library with the prototypes of include/splice_pages.h."""
    global _declared
    lib = S.load_library()
    if _declared is not lib:
        vp, i32, i64, size = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t
        shp, cal = ctypes.POINTER(S.SpliceShape), ctypes.POINTER(S.SpliceCall)
        pgs, rop = ctypes.POINTER(SplicePages), ctypes.POINTER(T.SpliceRope)
        for name, res, args in (
                ("splice_page_bytes", i64, [shp]),
                ("splice_page_append", i32, [shp, pgs, rop] + [vp] * 5 + [vp, i64] * 3 + [vp] * 3),
                ("splice_page_read", i32, [shp, pgs] + [vp] * 7),
                ("splice_page_attn_workspace_bytes", i64, [shp, cal, pgs]),
                ("splice_page_attn", i32, [shp, cal, pgs] + [vp] * 11 + [size, vp]),
                ("splice_page_fork", i32, [shp, pgs] + [vp] * 10 + [i64, vp]),
                ("splice_page_compact", i32, [shp, pgs] + [vp] * 4 + [i64, vp])):
            f = getattr(lib, name)
            f.restype, f.argtypes = res, args   # (a structure passes by reference where its pointer is declared)
        _declared = lib
    return lib


# ------------------------------------------------------------------ structs, checks

def make_pages(n_pages: int, table_len: int, n_tokens: int = 1) -> SplicePages:
    """Pools of ``n_pages`` pages, tables of ``table_len`` entries a cell, and T = ``n_tokens`` tokens a cell in a call."""
    return SplicePages(n_pages, table_len, n_tokens)


def splice_page_bytes(shape) -> int:
    """Bytes of one page of one layer."""
    return S._check(_library().splice_page_bytes(shape), "splice_page_bytes")


def _cells(shape, pages, cell_step, cell_new) -> Tuple[bytes, Optional[bytes]]:
    steps = T._steps(cell_step, shape.n_cells)
    return steps, None if cell_new is None else T._host(cell_new, shape.n_cells, 1, "cell_new", "entries")


def _tables(t, name: str, shape, pages, dev) -> int:
    return T._ptr(t, name, shape.n_cells * pages.table_len, S._torch.int32, dev)


def _pool(t, shape, pages, dev) -> int:
    return T._ptr(t, "pool", pages.n_pages * (68 * shape.n_kv_heads * shape.head_dim), S._torch.uint8, dev)


def _pools(t, shape, pages, dev) -> Tuple[int, int]:
    """(address, bytes from one layer to the next) of uint8 [n_layers][n_pages][page_bytes], each layer dense."""
    dims = (shape.n_layers, pages.n_pages, 68 * shape.n_kv_heads * shape.head_dim)
    if t is None or t.get_device() != dev[0]:
        raise ValueError(f"pools must be a tensor on {dev[1]}")
    if t.dtype is not S._torch.uint8:
        raise ValueError(f"pools has dtype {t.dtype}, expected {S._torch.uint8}")
    if t.shape != dims:
        raise ValueError(f"pools has shape {tuple(t.shape)}, expected {dims}")
    layer = dims[1] * dims[2]
    if not t[0].is_contiguous() or (dims[0] > 1 and t.stride(0) < layer):
        raise ValueError("pools: every layer must be dense and the layers apart")
    return t.data_ptr(), t.stride(0) if dims[0] > 1 else layer


# ------------------------------------------------------------------ C entry points

def splice_page_append(shape, pages, rope, freq, cell_step, cell_new, tables, q, k, v, q_out, pool, pos=None,
                       stream=None) -> None:
    """Rotate the tokens' ``q`` [C][T][Hq][D] into ``q_out`` and write their rotated ``k`` and their ``v``
    ([C][T][Hkv][D]) as rows s_c .. of the cells, in 4 bits (``cell_new``: how many of each cell, None for all T).
    ``q`` and ``q_out`` may both be None: then only rows are written."""
    lib = _library()
    dev = T._anchor(pool, "pool")
    n, C, t = pages.n_tokens, shape.n_cells, S._torch
    qo, qp, qs = None, None, 0
    if q is not None or q_out is not None:
        qo = T._ptr(q_out, "q_out", C * n * shape.n_q_heads * shape.head_dim, t.bfloat16, dev)
        qp, qs = T._rows(q, "q", shape, n, shape.n_q_heads, dev)
    kp, ks = T._rows(k, "k", shape, n, shape.n_kv_heads, dev)
    vp, vs = T._rows(v, "v", shape, n, shape.n_kv_heads, dev)
    tp, pl = _tables(tables, "tables", shape, pages, dev), _pool(pool, shape, pages, dev)
    pp = None if pos is None else T._ptr(pos, "pos", C * n, t.int64, dev)
    fp = None if rope.rotary_dim == 0 and freq is None else T._ptr(freq, "freq", rope.rotary_dim // 2, t.float64, dev)
    steps, new = _cells(shape, pages, cell_step, cell_new)
    S._check(lib.splice_page_append(shape, pages, rope, steps, new, tp, pp, fp, qp, qs, kp, ks, vp, vs, qo, pl,
                                    T._stream(stream, dev)), "splice_page_append")


def splice_page_read(shape, pages, cell_step, cell_new, tables, pool, rows_k, rows_v, stream=None) -> None:
    """``rows_k``, ``rows_v`` (bf16 [C][Hkv][T][D]): rows cell_step[c] + i of the cells, i < cell_new[c]."""
    lib = _library()
    dev = T._anchor(rows_k, "rows_k")
    n = shape.n_cells * shape.n_kv_heads * pages.n_tokens * shape.head_dim
    rk, rv = (T._ptr(x, name, n, S._torch.bfloat16, dev) for x, name in ((rows_k, "rows_k"), (rows_v, "rows_v")))
    tp, pl = _tables(tables, "tables", shape, pages, dev), _pool(pool, shape, pages, dev)
    steps, new = _cells(shape, pages, cell_step, cell_new)
    S._check(lib.splice_page_read(shape, pages, steps, new, tp, pl, rk, rv, T._stream(stream, dev)), "splice_page_read")


def splice_page_attn_workspace_bytes(shape, call, pages) -> int:
    return S._check(_library().splice_page_attn_workspace_bytes(shape, call, pages), "splice_page_attn_workspace_bytes")


def splice_page_attn(shape, call, pages, cell_LW, cell_step, cell_new, tables, clean_table, donor_table, q, pool, out, lse,
                     workspace, stream=None) -> None:
    """Spliced attention of every cell's tokens: ``out`` bf16 [C][T][Hq][D], ``lse`` float32 [C][T][Hq].

    ``clean_table``, ``donor_table``: int32 [ceil(T_p / 64)] pages of the prompt's slots (donor None for ZERO)."""
    lib = _library()
    dev = T._anchor(q, "q")
    t, C, n, Hq, D = S._torch, shape.n_cells, pages.n_tokens, shape.n_q_heads, shape.head_dim
    qp = T._ptr(q, "q", C * n * Hq * D, t.bfloat16, dev)
    tp, pl = _tables(tables, "tables", shape, pages, dev), _pool(pool, shape, pages, dev)
    n_prompt = -(-shape.prompt_len // SPLICE_PAGE_ROWS)
    cp = None if n_prompt == 0 and clean_table is None else T._ptr(clean_table, "clean_table", n_prompt, t.int32, dev)
    if shape.donor_kind == S.SPLICE_DONOR_ZERO:
        if donor_table is not None:
            raise ValueError("the ZERO donor takes no table")
        dp = None
    else:
        dp = None if n_prompt == 0 and donor_table is None else T._ptr(donor_table, "donor_table", n_prompt, t.int32, dev)
    op, lp = T._ptr(out, "out", C * n * Hq * D, t.bfloat16, dev), T._ptr(lse, "lse", C * n * Hq, t.float32, dev)
    wp, wbytes = T._workspace(workspace, dev)
    lwp = T._host(cell_LW, C, 2, "cell_LW", "rows")
    steps, new = _cells(shape, pages, cell_step, cell_new)
    S._check(lib.splice_page_attn(shape, call, pages, lwp, steps, new, tp, cp, dp, qp, pl, op, lp, wp, wbytes,
                                  T._stream(stream, dev)), "splice_page_attn")


def splice_page_fork(shape, pages, parent, rows, want, tables, refs, new_tables, new_refs, missing, copied, pools,
                     stream=None) -> None:
    """Cell c becomes the first ``rows[c]`` rows of cell ``parent[c]`` (-1: empty), with pages for ``want[c]`` rows: see
    include/splice_pages.h.  ``tables`` int32 [C][table_len] and ``refs`` int32 [n_pages] as they are, ``new_tables`` and
    ``new_refs`` as they become; ``missing`` int32 [1], ``copied`` int32 [C][2]; ``pools`` uint8
    [n_layers][n_pages][page_bytes]."""
    lib = _library()
    dev = T._anchor(tables, "tables")
    i32, C = S._torch.int32, shape.n_cells
    tp, np_ = _tables(tables, "tables", shape, pages, dev), _tables(new_tables, "new_tables", shape, pages, dev)
    rp, nr = T._ptr(refs, "refs", pages.n_pages, i32, dev), T._ptr(new_refs, "new_refs", pages.n_pages, i32, dev)
    mp, cp = T._ptr(missing, "missing", 1, i32, dev), T._ptr(copied, "copied", 2 * C, i32, dev)
    pl, stride = _pools(pools, shape, pages, dev)
    host = [T._host(x, C, 1, name, "entries") for x, name in ((parent, "parent"), (rows, "rows"), (want, "want"))]
    S._check(lib.splice_page_fork(shape, pages, *host, tp, rp, np_, nr, mp, cp, pl, stride, T._stream(stream, dev)),
             "splice_page_fork")


def splice_page_compact(shape, pages, cell_step, keep, tables, pools, stream=None) -> None:
    """Row cell_step[c] + i = row cell_step[c] + keep[c][i] in every layer of ``pools`` (``keep`` int32 [C][T], ascending, ended
    by -1)."""
    lib = _library()
    dev = T._anchor(keep, "keep")
    kp = T._ptr(keep, "keep", shape.n_cells * pages.n_tokens, S._torch.int32, dev)
    tp = _tables(tables, "tables", shape, pages, dev)
    pl, stride = _pools(pools, shape, pages, dev)
    S._check(lib.splice_page_compact(shape, pages, T._steps(cell_step, shape.n_cells), kp, tp, pl, stride,
                                     T._stream(stream, dev)), "splice_page_compact")


# ------------------------------------------------------------------ a sweep's cache

class PageCache:
    """The pages of C sweep cells and of the prompts that they share, for all layers: ``pools`` (uint8
    [n_layers][n_pages][page_bytes]), ``tables`` (int32, a row a cell), ``refs`` (int32 [n_pages]: who holds a page).

    A cell has pages for as many rows as ``fork`` or ``reserve`` last gave it (``rows``, on the host); the clean prompt's pages
    and the donor's are two rows more of the table, filled by ``load_prompt``.  The tensors stay where they are, so that
    captured calls keep working.  Calls go to the current stream."""

    def __init__(self, n_cells: int, n_layers: int, n_q_heads: int, n_kv_heads: int, head_dim: int, prompt_len: int, span,
                 capacity: int, n_pages: int, donor_zero: bool = False, device="cuda"):
        S.load_library()
        t = S._torch
        if n_cells + 2 > S.SPLICE_MAX_CELLS:
            raise ValueError(f"a cache has {S.SPLICE_MAX_CELLS - 2} cells at most, and its prompts")
        prompt = -(-prompt_len // SPLICE_PAGE_ROWS) * (1 if donor_zero else 2)
        if n_pages < prompt:
            raise ValueError(f"the prompts alone take {prompt} pages of {n_pages}")
        self.n_cells, self.capacity, self.prompt_len = n_cells, capacity, prompt_len
        self.table_len = max(-(-capacity // SPLICE_PAGE_ROWS), -(-prompt_len // SPLICE_PAGE_ROWS), 1)
        shape = lambda cells, layers, rows: S.make_shape(cells, layers, n_q_heads, n_kv_heads, head_dim, prompt_len, span,  # noqa: E731
                                                         rows, donor_zero, "bf16")
        self.shape = shape(n_cells, n_layers, capacity)                # of the cells
        self._every = shape(n_cells + 2, n_layers, self.table_len * SPLICE_PAGE_ROWS)
        self._row = shape(1, n_layers, self.table_len * SPLICE_PAGE_ROWS)
        with t.device(device):
            # (bytes that no row has filled are never looked at: clear them all the same, a pool is handed on)
            self.pools = t.zeros((n_layers, n_pages, splice_page_bytes(self.shape)), dtype=t.uint8, device=device)
            self._tables = t.full((n_cells + 2, self.table_len), -1, dtype=t.int32, device=device)
            self.refs = t.zeros(n_pages, dtype=t.int32, device=device)
            self._next = t.empty_like(self._tables), t.empty_like(self.refs)
            self.missing = t.zeros(1, dtype=t.int32, device=device)
            self._unseen = t.zeros_like(self.missing)                  # pages missing since the host last waited
            self.copied = t.zeros((n_cells + 2, 2), dtype=t.int32, device=device)
        self._prompts = [prompt_len, 0 if donor_zero else prompt_len]
        self._held = [0, 0]                                            # rows of the prompts that have pages
        self.rows = np.zeros(n_cells, np.int32)                        # rows of the cells that have pages
        self._lost = np.zeros(n_cells, bool)                           # cells without some of the rows that they took over
        self._all = np.iinfo(np.int32).max
        self._common = np.diag(np.full(n_cells, self._all, np.int32))  # pages that two cells share: the first ones of both
        self._shared = np.zeros(n_cells, np.int32)                     # rows of the pages that a cell shares
        self.fork(np.full(n_cells, -1), self.rows, self.rows)

    @property
    def tables(self):
        """The cells' tables (int32 [C][table_len])."""
        return self._tables[:self.n_cells]

    @property
    def clean_table(self):
        return self._tables[self.n_cells, :-(-self.prompt_len // SPLICE_PAGE_ROWS)]

    @property
    def donor_table(self):
        """The donor's pages; None for ZERO."""
        if self.shape.donor_kind == S.SPLICE_DONOR_ZERO:
            return None
        return self._tables[self.n_cells + 1, :-(-self.prompt_len // SPLICE_PAGE_ROWS)]

    def pages(self, n_tokens: int) -> SplicePages:
        return make_pages(self.pools.shape[1], self.table_len, n_tokens)

    def fork(self, parent, rows, want=None) -> None:
        """Cell c goes on from the first ``rows[c]`` rows of cell ``parent[c]`` (-1: from none), with pages for ``want[c]`` rows
        (``rows`` without): ``splice_page_fork``.  ``missing`` says how many pages there were too few, ``copied`` which were.

        Where pages were too few a cell has those up to its first absent one, and ``rows`` says so: ask again when others have
        given theirs back.  A cell for which the copy of a page in use was among them has lost that page's rows
        (``rows`` is below what it was to take over).  To know this the host waits for a call that asks for pages.  It does not
        for a captured one: that is taken to find them all, and what its replays missed is noticed behind the next call that is
        waited for (as is the copy of a page that ``refs`` was raised for by hand)."""
        want = rows if want is None else want
        C = self.n_cells
        cells = [np.asarray(x, dtype=np.int32).reshape(-1) for x in (parent, rows, want)]
        if any(len(x) != C for x in cells):
            raise ValueError(f"parent, rows and want have an entry for each of the {C} cells")
        if (cells[0] >= C).any():
            raise ValueError(f"a parent is one of the {C} cells, or negative")
        if C and cells[2].max() > self.capacity:
            raise ValueError(f"a cell has {self.capacity} rows at most")
        if (cells[1] > self.rows[np.maximum(cells[0], 0)])[cells[0] >= 0].any():
            raise ValueError("a cell cannot take over more rows than its parent has pages for")
        more = [C, C + 1], self._held, self._prompts
        host = [np.concatenate([x, np.asarray(y, dtype=np.int32)]) for x, y in zip(cells, more)]
        splice_page_fork(self._every, self.pages(1), *host, self._tables, self.refs, *self._next, self.missing, self.copied,
                         self.pools)
        self._tables.copy_(self._next[0])
        self.refs.copy_(self._next[1])
        self._unseen += self.missing
        self._held, self.rows = list(self._prompts), cells[2].copy()
        self._lost[:] = False
        # a page is asked for behind the rows that a cell takes over, or for the copy of their last one, if it is not its own
        parent, whole, part = cells[0], cells[1] // SPLICE_PAGE_ROWS, cells[1] % SPLICE_PAGE_ROWS > 0
        own = ((cells[1] == 0) | (parent == np.arange(C)) & (cells[1] >= self._shared)).all()
        asks = (-(-cells[2] // SPLICE_PAGE_ROWS) > (whole + part if own else whole)).any()
        self._share(parent, whole)
        if asks and not (self._tables.is_cuda and S._torch.cuda.is_current_stream_capturing()) and int(self._unseen) > 0:
            self._unseen.zero_()
            # a cell's pages are given from the first on, so what it has ends at the first absent one
            tables = self.tables.cpu().numpy()
            there = np.cumprod((tables >= 0) & (tables < self.pools.shape[1]), axis=1).sum(axis=1)
            self.rows = np.minimum(self.rows, there * SPLICE_PAGE_ROWS).astype(np.int32)
            self._lost = self.rows < cells[1]

    def _share(self, parent, whole) -> None:
        """Cells have taken over ``whole[c]`` full pages of cell ``parent[c]``; all others of a cell are its own."""
        if not self._shared.any() and np.bincount(parent[whole > 0], minlength=1).max() <= 1:
            return   # none are shared, and no two cells took over those of one
        of = np.maximum(parent, 0)
        common = self._common.take(of, axis=0).take(of, axis=1)   # (of a cell with itself: all)
        np.minimum(common, whole, out=common)
        np.minimum(common, whole[:, None], out=common)
        np.fill_diagonal(common, 0)
        self._shared = common.max(axis=1, initial=0) * np.int32(SPLICE_PAGE_ROWS)
        np.fill_diagonal(common, self._all)
        self._common = common

    def reserve(self, want) -> None:
        """Pages for ``want[c]`` rows of every cell; rows that it has stay.  A cell that has lost rows is given none behind
        those that it has: fork it, from these or from others."""
        want = np.asarray(want, dtype=np.int32).reshape(-1)
        if len(want) == self.n_cells and (self._lost & (want > self.rows)).any():
            raise ValueError(f"cells {np.flatnonzero(self._lost & (want > self.rows)).tolist()} have lost rows: fork them anew")
        lost = self._lost.copy()
        self.fork(np.arange(self.n_cells), np.minimum(want, self.rows), want)
        self._lost |= lost

    def _check_rows(self, steps, count) -> None:
        """That every cell may write rows steps[c] .. steps[c] + count[c] - 1 (host arrays; none where the step is negative or the
        count 0): they have pages, and no other cell has them too."""
        end = steps + np.asarray(count, dtype=np.int64)
        bad = (steps >= 0) & (end > steps) & (end > self.rows)
        if bad.any():
            c = int(np.flatnonzero(bad)[0])
            raise ValueError(f"cell {c} has pages for {self.rows[c]} rows, its tokens end at row {end[c]}: reserve them first")
        self._check_own(steps, end > steps)

    def _check_own(self, steps, writes) -> None:
        bad = (steps >= 0) & (steps < self._shared) & writes
        if bad.any():
            c = int(np.flatnonzero(bad)[0])
            raise ValueError(f"cell {c} shares its rows below {self._shared[c]} with other cells, so row {steps[c]} is not written: fork "
                             "the cell from the rows before it")

    def load_prompt(self, layer: int, k, v, donor: bool = False) -> None:
        """Rows of the clean prompt's (or the donor's) pages of a layer from bf16 [Hkv][T_p][D]."""
        t, sh = S._torch, self.shape
        dims = (sh.n_kv_heads, self.prompt_len, sh.head_dim)
        if tuple(k.shape) != dims or tuple(v.shape) != dims:
            raise ValueError(f"a prompt's k and v have shape {dims}")
        if donor and sh.donor_kind == S.SPLICE_DONOR_ZERO:
            raise ValueError("the ZERO donor has no rows")
        table = self._tables[self.n_cells + bool(donor)]
        rope = T.make_rope("half", 0)
        for a in range(0, self.prompt_len, SPLICE_MAX_PAGE_TOKENS):
            n = min(SPLICE_MAX_PAGE_TOKENS, self.prompt_len - a)
            part = [x[:, a:a + n].transpose(0, 1).contiguous()[None] for x in (k, v)]
            splice_page_append(self._row, self.pages(n), rope, None, [a], None, table, None, *part, None, self.pools[layer])

    def compact(self, cell_step, keep) -> None:
        """Row cell_step[c] + i of the cells = row cell_step[c] + keep[c][i] (``keep`` int32 [C][T] on the device): the tokens
        that were accepted, or that an eviction leaves.  A cell_step[c] in a page that other cells have too is refused (a fork
        shares the full pages of the rows that it takes over): ``fork`` the cell from its first cell_step[c] rows, or give -1."""
        self._check_own(S._steps(cell_step, self.n_cells)[0], True)
        splice_page_compact(self.shape, self.pages(keep.shape[1]), cell_step, keep, self.tables, self.pools)
